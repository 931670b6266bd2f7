"""The gated feed-forward part and its gradients against plain torch in 64 bits."""
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


def inputs(rows, ff, d, dtype, seed=0, spread=1.5):
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.randn((rows, d), generator=g, device="cuda").to(dtype)
    wg, wu = ((spread * d ** -0.5 * torch.randn((ff, d), generator=g, device="cuda")).to(dtype) for _ in range(2))
    return x, wg, wu, torch.randn((rows, ff), generator=g, device="cuda").to(dtype)


def check(ops, x, wg, wu, gy, kind):
    out = ops.gated_feed_forward(x, wg, wu, kind)
    want, bound, _ = ref.gated(x, wg, wu, kind)
    assert out.dtype is x.dtype and out.is_contiguous()
    near(out, want, bound, "out")
    got = ops.gated_feed_forward_grad(x, wg, wu, gy, kind)
    parts = 2 if x.shape[0] <= 128 or wg.shape[0] <= 32 else 1        # (a CTA a tile)
    for v, (want, bound), what in zip(got, ref.gated_grad(x, wg, wu, gy, kind, parts), ("d_x", "d_w_gate", "d_w_up")):
        assert v.dtype is x.dtype and v.is_contiguous()
        near(v, want, bound, what)
    return out, got


@pytest.mark.parametrize("dtype,kind", [(BF16, "silu"), (F16, "silu"), (BF16, "gelu"), (F16, "gelu")])
@pytest.mark.parametrize("rows,ff,d", [(1, 1, 8), (1, 64, 64), (5, 33, 72), (8, 4096, 256), (16, 1000, 768), (33, 250, 512), (96, 2051, 128), (128, 64, 24), (129, 33, 64), (129, 31, 72),
                                       (200, 64, 1024), (256, 256, 96), (300, 515, 768), (513, 130, 320), (1000, 2000, 1024), (2049, 100, 136), (7, 130, 1032), (100, 70, 1272)])
def test_sizes(ops, dtype, kind, rows, ff, d):
    check(ops, *inputs(rows, ff, d, dtype, seed=rows + ff + d), kind)


@pytest.mark.parametrize("kind", ["silu", "gelu"])
@pytest.mark.parametrize("rows", [4, 300])
def test_gates_of_any_size(ops, kind, rows):
    """Far below zero the activation vanishes, far above it is the gate itself."""
    x, wg, wu, gy = inputs(rows, 200, 64, BF16, seed=1, spread=40.0)
    check(ops, x, wg, wu, gy, kind)


@pytest.mark.parametrize("size", [2.0 ** -20, 1e-4, 300.0])
@pytest.mark.parametrize("rows", [6, 260])
def test_gradients_of_any_size_in_fp16(ops, size, rows):
    x, wg, wu, gy = inputs(rows, 150, 64, F16, seed=2)
    gy = (gy.float() * size).half()
    for v, (want, bound) in zip(ops.gated_feed_forward_grad(x, wg, wu, gy), ref.gated_grad(x, wg, wu, gy, "silu")):
        sure = want.abs() + bound < 65000
        near(torch.where(sure, v.double(), 0.0), torch.where(sure, want, 0.0), bound, "gradient")


@pytest.mark.parametrize("rows", [6, 300])
def test_shapes_strides_and_slices(ops, rows):
    x, wg, wu, gy = inputs(rows, 120, 64, BF16, seed=3)
    out = ops.gated_feed_forward(x, wg, wu)
    grads = ops.gated_feed_forward_grad(x, wg, wu, gy)
    assert torch.equal(ops.gated_feed_forward(x.view(2, rows // 2, 64), wg, wu), out.view(2, rows // 2, 120))
    for v, y in zip(ops.gated_feed_forward_grad(x.view(2, rows // 2, 64), wg, wu, gy.view(2, rows // 2, 120)), grads):
        assert torch.equal(v.reshape(y.shape), y)
    assert torch.equal(ops.gated_feed_forward(x[0], wg, wu), ops.gated_feed_forward(x[:1], wg, wu)[0])
    both = torch.cat([wg, wu])                     # side by side, as some keep them
    wide = torch.full((rows, 3, 64), math.nan, device="cuda", dtype=BF16)
    wide[:, 1] = x
    g2 = torch.full((rows, 125), math.nan, device="cuda", dtype=BF16)
    g2[:, 3:123] = gy                              # rows of odd length, at odd places
    assert torch.equal(ops.gated_feed_forward(wide[:, 1], both[:120], both[120:]), out)
    for v, y in zip(ops.gated_feed_forward_grad(wide[:, 1], both[:120], both[120:], g2[:, 3:123]), grads):
        assert torch.equal(v, y)
    one = torch.full((1, 1), 0.5, device="cuda", dtype=BF16).expand(rows, 120).contiguous()
    row = one[:1].expand(rows, 120)                # the same row for all
    for v, y in zip(ops.gated_feed_forward_grad(x, wg, wu, row), ops.gated_feed_forward_grad(x, wg, wu, one)):
        assert torch.equal(v, y)


@pytest.mark.parametrize("rows,ff", [(7, 123), (300, 123), (300, 128), (2047, 2051)])
@pytest.mark.parametrize("size", [1.0, 2.0 ** -14])
def test_gradients_in_fp16_lie_anywhere(ops, rows, ff, size):
    """The largest gradient is looked for where the rows are: at odd places, of odd length, the same row for all; what lies between them is not looked at."""
    x, wg, wu, gy = inputs(rows, ff, 64, F16, seed=20)
    gy = (gy.float() * size).half()
    want = ops.gated_feed_forward_grad(x, wg, wu, gy)
    for v, (w, b) in zip(want, ref.gated_grad(x, wg, wu, gy, "silu")):
        near(v, w, b, "gradient")
    for left, right in ((0, 5), (3, 2), (8, 8)):
        g2 = torch.full((rows, left + ff + right), 60000.0, device="cuda", dtype=F16)
        g2[:, left:left + ff] = gy
        for v, y in zip(ops.gated_feed_forward_grad(x, wg, wu, g2[:, left:left + ff]), want):
            assert torch.equal(v, y)
    row = gy[:1].expand(rows, ff)
    for v, y in zip(ops.gated_feed_forward_grad(x, wg, wu, row), ops.gated_feed_forward_grad(x, wg, wu, row.contiguous())):
        assert torch.equal(v, y)


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("rows,ff,d", [(9000, 40, 72), (9001, 130, 128), (20, 20011, 64), (300, 20001, 128), (20001, 4, 8)])
def test_long_sums_of_few_tiles(ops, dtype, rows, ff, d):
    """Sums that are cut into many, of either kind of gradient."""
    check(ops, *inputs(rows, ff, d, dtype, seed=21), "silu")


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("rows", [5, 280])
def test_infinities_and_nan_stay_in_their_rows(ops, dtype, rows):
    x, wg, wu, gy = inputs(rows, 90, 64, dtype, seed=4)
    out = ops.gated_feed_forward(x, wg, wu)
    d_x = ops.gated_feed_forward_grad(x, wg, wu, gy)[0]
    x2, gy2 = x.clone(), gy.clone()
    x2[1, 5] = math.nan
    gy2[2, 7] = math.nan
    got, d = ops.gated_feed_forward(x2, wg, wu), ops.gated_feed_forward_grad(x2, wg, wu, gy2)[0]
    assert got[1].isnan().all() and d[1].isnan().all() and d[2].isnan().all()
    keep = torch.arange(rows, device="cuda") != 1
    assert torch.equal(got[keep], out[keep])
    keep &= torch.arange(rows, device="cuda") != 2
    assert torch.equal(d[keep], d_x[keep])
    w2 = wg.clone()
    w2[3, 0] = math.inf
    got = ops.gated_feed_forward(x, w2, wu)
    keep = torch.arange(90, device="cuda") != 3
    assert torch.equal(got[:, keep], out[:, keep])
    up = x[:, 0] > 0
    assert torch.equal(got[up, 3].isinf(), torch.ones_like(got[up, 3], dtype=torch.bool)) and got[x[:, 0] < 0, 3].isnan().all()


def test_empty_calls_and_what_is_needed(ops):
    x, wg, wu, gy = inputs(300, 70, 64, BF16, seed=5)
    assert ops.gated_feed_forward(x[:0], wg, wu).shape == (0, 70)
    d = ops.gated_feed_forward_grad(x[:0], wg, wu, gy[:0])
    assert d[0].shape == (0, 64) and (d[1] == 0).all() and (d[2] == 0).all()
    all_ = ops.gated_feed_forward_grad(x, wg, wu, gy)
    for need in ((True, False, False), (False, True, True), (False, True, False), (False, False, True), (False, False, False)):
        for v, y, n in zip(ops.gated_feed_forward_grad(x, wg, wu, gy, need=need), all_, need):
            assert v is None if not n else torch.equal(v, y)


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("kind", ["silu", "gelu"])
@pytest.mark.parametrize("rows", [4, 300])
def test_autograd_and_differences(ops, dtype, kind, rows):
    g = torch.Generator(device="cuda").manual_seed(6)
    x = (torch.randint(-12, 13, (rows, 64), generator=g, device="cuda") / 8).to(dtype).requires_grad_()
    wg, wu = ((torch.randint(-12, 13, (96, 64), generator=g, device="cuda") / 64).to(dtype).requires_grad_() for _ in range(2))
    gy = torch.randn((rows, 96), generator=g, device="cuda").to(dtype)
    leaves = [x, wg, wu]
    d = torch.autograd.grad(ops.gated_feed_forward(x, wg, wu, kind), leaves, gy)
    with torch.no_grad():
        for v, y in zip(ops.gated_feed_forward_grad(x, wg, wu, gy, kind), d):
            assert torch.equal(v, y)
        exact = ref.gated_grad(x, wg, wu, gy, kind)
        for i, step in ((0, 0.125), (1, 1 / 64), (2, 1 / 64)):
            v = torch.randint(-1, 2, leaves[i].shape, generator=g, device="cuda").double()

            def at(s):
                a = [(t + s * step * v).to(dtype) if j == i else t for j, t in enumerate(leaves)]
                want, bound, _ = ref.gated(*a, kind)
                return (ops.gated_feed_forward(*a, kind).double() * gy).sum(), (want * gy).sum(), (bound * gy.abs()).sum()
            plus, minus = at(1), at(-1)
            slope, own = (plus[0] - minus[0]) / (2 * step), ((plus[1] - minus[1]) / (2 * step) - (exact[i][0] * v).sum()).abs()
            assert abs(slope - (d[i].double() * v).sum()) <= own + (plus[2] + minus[2]) / (2 * step) + (exact[i][1] * v.abs()).sum()
    # the gradient of a sum comes as one number for all places
    for v, y in zip(torch.autograd.grad(ops.gated_feed_forward(x, wg, wu, kind).sum(), leaves), ops.gated_feed_forward_grad(*(t.detach() for t in leaves), torch.ones_like(gy), kind)):
        assert torch.equal(v, y)
    only = torch.autograd.grad(ops.gated_feed_forward(x.detach(), wg.detach(), wu, kind), wu, gy)[0]
    assert torch.equal(only, d[2])


@pytest.mark.parametrize("rows", [5, 300])
def test_streams_graphs_and_repeats(ops, rows):
    x, wg, wu, gy = inputs(rows, 515, 256, F16, seed=7)
    want = [ops.gated_feed_forward(x, wg, wu), *ops.gated_feed_forward_grad(x, wg, wu, gy)]
    other = inputs(rows, 515, 256, F16, seed=8)
    want2 = [ops.gated_feed_forward(*other[:3]), *ops.gated_feed_forward_grad(*other)]
    static = [t.clone() for t in (x, wg, wu, gy)]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        cap = [ops.gated_feed_forward(*static[:3]), *ops.gated_feed_forward_grad(*static)]
    outs, sides = [], [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    for _ in range(8):
        for s in sides:
            with torch.cuda.stream(s):
                outs.append([ops.gated_feed_forward(x, wg, wu), *ops.gated_feed_forward_grad(x, wg, wu, gy)])
    graph.replay()
    torch.cuda.synchronize()
    for got in outs + [cap]:
        assert all(torch.equal(v, y) for v, y in zip(got, want))
    for a, b in zip(static, other):
        a.copy_(b)
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(v, y) for v, y in zip(cap, want2))


def test_offsets_beyond_32_bits(ops):
    rows, ff = 66_003, 33_001
    x, wg, wu, _ = inputs(rows, ff, 64, BF16, seed=9)
    out = ops.gated_feed_forward(x, wg, wu)
    for r in (slice(0, 3), slice(40_000, 40_003), slice(rows - 3, rows)):
        want, bound, _ = ref.gated(x[r], wg, wu, "silu")
        near(out[r], want, bound, "out")


@pytest.mark.parametrize("rows", [5, 300])
def test_a_wait_that_runs_out_is_told(ops, rows):
    x, wg, wu, gy = inputs(rows, 200, 256, BF16, seed=10)
    want = [ops.gated_feed_forward(x, wg, wu), *ops.gated_feed_forward_grad(x, wg, wu, gy)]
    from paper_2507_23777_b200 import binding
    lib = binding.load()
    try:
        lib.xsm_debug_product_waits(2000, 1)
        for f in (lambda: ops.gated_feed_forward(x, wg, wu), lambda: ops.gated_feed_forward_grad(x, wg, wu, gy)):
            f()
            with pytest.raises(binding.XsmError, match="patience"):
                ops.check()
    finally:
        lib.xsm_debug_product_waits(0, 0)
    got = [ops.gated_feed_forward(x, wg, wu), *ops.gated_feed_forward_grad(x, wg, wu, gy)]
    ops.check()
    assert all(torch.equal(v, y) for v, y in zip(got, want))


def test_refusals(ops):
    x, wg, wu, gy = inputs(4, 100, 64, BF16)
    odd = torch.zeros(4 * 64 + 1, dtype=BF16, device="cuda")[1:].view(4, 64)
    for bad in (dict(x=x.float(), w_gate=wg.float(), w_up=wu.float()), dict(w_up=wu.half()), dict(w_up=wu[:99]), dict(x=x[:, :60], w_gate=wg[:, :60], w_up=wu[:, :60]), dict(w_gate=wg[:, :56], w_up=wu[:, :56]),
                dict(w_gate=wg[:0], w_up=wu[:0]), dict(x=x.cpu()), dict(w_gate=wg.cpu(), w_up=wu.cpu()), dict(activation="tanh"), dict(activation=None), dict(x=odd),
                dict(x=x[:1].expand(4, 64)), dict(w_gate=wg.T, w_up=wu.T)):
        args = dict(x=x, w_gate=wg, w_up=wu)
        args.update(bad)
        with pytest.raises((ValueError, RuntimeError)):
            ops.gated_feed_forward(**args)
        with pytest.raises((ValueError, RuntimeError)):
            ops.gated_feed_forward_grad(**args, grad=gy)
    for bad in (gy[:3], gy.half(), gy.cpu(), gy.T.contiguous().T):
        with pytest.raises(ValueError):
            ops.gated_feed_forward_grad(x, wg, wu, bad)
    xg = x.clone().requires_grad_()
    with pytest.raises(ValueError, match="no_grad"):
        ops.gated_feed_forward_grad(xg, wg, wu, gy)
    (g1,) = torch.autograd.grad(ops.gated_feed_forward(xg, wg, wu).sum(), xg, create_graph=True)
    with pytest.raises(RuntimeError):
        torch.autograd.grad(g1.float().sum(), xg)
    with torch.autograd.forward_ad.dual_level():
        with pytest.raises(ValueError, match="forward-mode"):
            ops.gated_feed_forward(torch.autograd.forward_ad.make_dual(x, x.clone()), wg, wu)
