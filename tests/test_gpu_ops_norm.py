"""Norms of heads with the rotation of the positions, their gradients, and the same into a paged cache, against plain torch in 64 bits."""
import math

import pytest
import torch

import block_reference as ref
from block_reference import BF16, F16, F32, near

pytestmark = pytest.mark.gpu

EPS = 1e-6


@pytest.fixture(scope="module")
def ops():
    assert torch.cuda.is_available(), "this test needs a B200"
    from paper_2507_23777_b200 import build, ops
    build.build()
    return ops


def inputs(batch, m, heads, kv_heads, d, dtype, seed=0, gain_t=F32):
    g = torch.Generator(device="cuda").manual_seed(seed)
    qkv = torch.randn((batch, m, heads + 2 * kv_heads, d), generator=g, device="cuda")
    qkv = (qkv * torch.exp(torch.randn((1, 1, heads + 2 * kv_heads, 1), generator=g, device="cuda"))).to(dtype)
    q, k, v = qkv.split([heads, kv_heads, kv_heads], 2)
    gains = [(1 + 0.2 * torch.randn(d, generator=g, device="cuda")).to(gain_t) for _ in range(2)]
    grads = [torch.randn((batch, m, n, d), generator=g, device="cuda").to(dtype) for n in (heads, kv_heads)]
    return q, k, v, gains, grads


def check(ops, q, k, gains, grads, rope=None, positions=None, eps=EPS, interleaved=False):
    out = ops.norm_rotate(q, k, *gains, rope=rope, positions=positions, eps=eps, interleaved=interleaved)
    got = ops.norm_rotate_grad(q, k, *gains, *grads, rope=rope, positions=positions, eps=eps, interleaved=interleaved)
    for i, (x, gain, g) in enumerate(zip((q, k), gains, grads)):
        want, bound = ref.norm(x, gain, rope, positions, eps, interleaved)
        assert out[i].dtype is x.dtype
        near(out[i], want, bound, "qk"[i])
        (dx, b), (dg, c) = ref.norm_grad(x, gain, g, rope, positions, eps, interleaved)
        near(got[i], dx, b, "d_" + "qk"[i])
        assert got[2 + i].dtype is gain.dtype
        near(got[2 + i], dg, c, f"d_{'qk'[i]}_gain")
    return out, got


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("d", [32, 64, 96, 128, 256])
@pytest.mark.parametrize("interleaved", [False, True])
def test_types_widths_and_rotations(ops, dtype, d, interleaved):
    for rot in (d, d // 2, 2, 0, d - 2):
        rope = ops.rope_table(40, rot) if rot else None
        q, k, _, gains, grads = inputs(2, 19, 6, 2, d, dtype, seed=d + rot)
        check(ops, q, k, gains, grads, rope, interleaved=interleaved)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("batch,m,heads,kv_heads", [(1, 1, 1, 1), (1, 5, 16, 16), (3, 1, 32, 8), (1, 1, 7, 1), (5, 33, 12, 3), (2, 700, 9, 9), (64, 3, 28, 4), (1, 2100, 16, 2)])
def test_layouts_and_lengths(ops, dtype, batch, m, heads, kv_heads):
    q, k, _, gains, grads = inputs(batch, m, heads, kv_heads, 64, dtype, seed=m)
    check(ops, q, k, gains, grads, ops.rope_table(m, 64))


@pytest.mark.parametrize("dtype,gain_t", [(BF16, BF16), (F16, F16), (F32, BF16), (BF16, F16)])
def test_gains_of_any_type(ops, dtype, gain_t):
    q, k, _, gains, grads = inputs(2, 30, 4, 2, 128, dtype, seed=1, gain_t=gain_t)
    check(ops, q, k, gains, grads, ops.rope_table(30, 64))


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("rot", [64, 6])
def test_positions(ops, dtype, rot):
    """Any order, the same twice, and those that the rope does not have: zero, without a gradient."""
    q, k, _, gains, grads = inputs(3, 50, 4, 2, 64, dtype, seed=2)
    rope = ops.rope_table(100, rot)
    pos = torch.randint(0, 100, (3, 50), device="cuda", dtype=torch.int32)
    pos[0, 3], pos[1, 4], pos[2, 5], pos[0, 6] = -1, 100, 2 ** 31 - 1, -2 ** 31
    out, got = check(ops, q, k, gains, grads, rope, pos)
    for b, j in ((0, 3), (1, 4), (2, 5), (0, 6)):
        assert all((x[b, j] == 0).all() for x in (*out, *got[:2]))
    q2 = q.clone()
    q2[0, 3] = math.nan                      # in a token that has no place: nowhere else
    out2, got2 = ops.norm_rotate(q2, k, *gains, rope=rope, positions=pos), ops.norm_rotate_grad(q2, k, *gains, *grads, rope=rope, positions=pos)
    assert torch.equal(out2[0], out[0]) and all(torch.equal(x, y) for x, y in zip(got2, got))
    # without a rope positions do not matter
    assert all(torch.equal(x, y) for x, y in zip(ops.norm_rotate(q, k, *gains, positions=pos), ops.norm_rotate(q, k, *gains)))


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
def test_one_tensor_alone_and_empty_calls(ops, dtype):
    q, k, _, gains, grads = inputs(2, 21, 6, 3, 96, dtype, seed=3)
    rope = ops.rope_table(21, 96)
    both = ops.norm_rotate(q, k, *gains, rope=rope)
    g = ops.norm_rotate_grad(q, k, *gains, *grads, rope=rope)
    a, none = ops.norm_rotate(q, None, gains[0], None, rope=rope)
    none2, b = ops.norm_rotate(None, k, None, gains[1], rope=rope)
    assert none is None and none2 is None and torch.equal(a, both[0]) and torch.equal(b, both[1])
    x = ops.norm_rotate_grad(q, None, gains[0], None, grads[0], None, rope=rope)
    y = ops.norm_rotate_grad(None, k, None, gains[1], None, grads[1], rope=rope)
    assert x[1] is x[3] is y[0] is y[2] is None and torch.equal(x[0], g[0]) and torch.equal(y[1], g[1])
    for v, (w, bound) in ((x[2], ref.norm_grad(q, gains[0], grads[0], rope, None, EPS, False)[1]), (y[3], ref.norm_grad(k, gains[1], grads[1], rope, None, EPS, False)[1])):
        near(v, w, bound, "gain")
    e = ops.norm_rotate(q[:, :0], k[:, :0], *gains, rope=rope)
    assert e[0].shape == (2, 0, 6, 96) and e[1].shape == (2, 0, 3, 96)
    e = ops.norm_rotate_grad(q[:, :0], k[:, :0], *gains, grads[0][:, :0], grads[1][:, :0], rope=rope)
    assert e[0].shape == (2, 0, 6, 96) and (e[2] == 0).all() and (e[3] == 0).all()


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("interleaved", [False, True])
def test_rows_of_any_stride_and_alignment(ops, dtype, interleaved):
    q, k, _, gains, grads = inputs(2, 17, 4, 2, 64, dtype, seed=4)
    rope = ops.rope_table(17, 64)
    want, g = check(ops, q, k, gains, grads, rope, interleaved=interleaved)
    for shift in (1, 3):
        q2, gq2 = (torch.full((2, 17, 4, 64 + 5), math.nan, device="cuda", dtype=dtype) for _ in range(2))
        q2[..., shift:shift + 64], gq2[..., shift:shift + 64] = q, grads[0]
        out, got = check(ops, q2[..., shift:shift + 64], k, gains, [gq2[..., shift:shift + 64], grads[1]], rope, interleaved=interleaved)
    swapped = q.transpose(1, 2).contiguous().transpose(1, 2)            # [batch, heads, m, d] underneath
    assert torch.equal(ops.norm_rotate(swapped, k, *gains, rope=rope, interleaved=interleaved)[0], want[0])
    one = q[:1].expand(2, -1, -1, -1)                                   # the same rows for every sequence
    assert torch.equal(ops.norm_rotate(one, None, gains[0], None, rope=rope)[0], ops.norm_rotate(one.contiguous(), None, gains[0], None, rope=rope)[0])


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_rows_that_overlap(ops, dtype):
    """Windows of a longer row, a step of one element apart; and the same head for all.  (Rows that are not aligned have a kernel of their own, which adds the 64 squares up
    two a lane where the other has 8 or 16: equal within NORM's count of roundings, not bit by bit.)"""
    g = torch.Generator(device="cuda").manual_seed(30)
    base = torch.randn(4000, generator=g, device="cuda").to(dtype)
    rope = ops.rope_table(33, 64)
    gain, grad = torch.randn(64, generator=g, device="cuda"), torch.randn((2, 33, 3, 64), generator=g, device="cuda").to(dtype)
    for strides in ((1000, 1, 300, 1), (0, 1, 0, 1), (1, 64, 0, 1), (0, 0, 0, 1)):
        x = base.as_strided((2, 33, 3, 64), strides)
        out = ops.norm_rotate(x, None, gain, None, rope=rope)[0]
        near(out, *ref.norm(x, gain, rope, None, 1e-6, False), "norm")
        d, _, d_gain, _ = ops.norm_rotate_grad(x, None, gain, None, grad, None, rope=rope)
        (dx, b), (dg, bg) = ref.norm_grad(x, gain, grad, rope, None, 1e-6, False)
        near(d, dx, b, "dx")
        near(d_gain, dg, bg, "d_gain")
        assert out.stride(3) == 1 == d.stride(3)


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
def test_zero_large_and_odd_rows(ops, dtype):
    q, k, _, gains, grads = inputs(1, 8, 2, 2, 64, dtype, seed=5)
    q, k = q.clone(), k.clone()
    q[0, 0] = 0
    q[0, 1] *= 1e-4
    q[0, 2] *= 50
    rope = ops.rope_table(8, 64)
    check(ops, q, k, gains, grads, rope)
    check(ops, q[:, 1:], k[:, 1:], gains, [g[:, 1:] for g in grads], rope, eps=0.0)
    clean = ops.norm_rotate(q, k, *gains, rope=rope)
    q[0, 3, 1, 7] = math.nan
    out = ops.norm_rotate(q, k, *gains, rope=rope)
    assert out[0][0, 3, 1].isnan().all()
    out[0][0, 3, 1] = clean[0][0, 3, 1]
    assert torch.equal(out[0], clean[0])


@pytest.mark.parametrize("rot,interleaved", [(64, False), (32, True)])
def test_autograd_and_differences(ops, rot, interleaved):
    q, k, _, gains, grads = inputs(2, 9, 3, 2, 64, F32, seed=6)
    rope = ops.rope_table(30, rot)
    pos = torch.randint(0, 30, (2, 9), device="cuda", dtype=torch.int32)
    leaves = [t.clone().requires_grad_() for t in (q, k, *gains)]
    more = dict(rope=rope, positions=pos, interleaved=interleaved)
    out = ops.norm_rotate(*leaves, **more)
    d = torch.autograd.grad(out, leaves, grads)
    with torch.no_grad():
        for x, y in zip(ops.norm_rotate_grad(*leaves, *grads, **more), d):
            assert torch.equal(x, y)
        g = torch.Generator(device="cuda").manual_seed(7)
        for i, t in enumerate(leaves):
            v = torch.randn(t.shape, generator=g, device="cuda")
            step = 2.0 ** -7

            def at(s):
                a = [u + s * step * v if j == i else u for j, u in enumerate(leaves)]
                kernel = sum((o.double() * w).sum() for o, w in zip(ops.norm_rotate(*a, **more), grads))
                exact = [ref.norm(x, gain, rope, pos, EPS, interleaved) for x, gain in zip(a[:2], a[2:])]
                return kernel, sum((e[0] * w).sum() for e, w in zip(exact, grads)), sum((e[1] * w.abs()).sum() for e, w in zip(exact, grads))
            plus, minus = at(1), at(-1)
            (dx, bx), (dg, bg) = ref.norm_grad(leaves[i % 2], leaves[2 + i % 2], grads[i % 2], rope, pos, EPS, interleaved)
            e, b = (dx, bx) if i < 2 else (dg, bg)
            slope, own = (plus[0] - minus[0]) / (2 * step), ((plus[1] - minus[1]) / (2 * step) - (e * v).sum()).abs()
            assert abs(slope - (d[i].double() * v).sum()) <= own + (plus[2] + minus[2]) / (2 * step) + (b * v.abs()).sum()
            assert own < 0.05 * (e * v).abs().sum()
    # only one of the results is used; only some of the leaves want a gradient
    (x,) = torch.autograd.grad((ops.norm_rotate(*leaves, **more)[0] * grads[0]).sum(), leaves[0])
    assert torch.equal(x, d[0])
    gains_only = [q, k, leaves[2], leaves[3]]
    for x, y in zip(torch.autograd.grad(ops.norm_rotate(*gains_only, **more), leaves[2:], grads), d[2:]):
        assert torch.equal(x, y)
    # a sum's gradient is one number for all places
    ones = [torch.ones_like(t) for t in grads]
    for x, y in zip(torch.autograd.grad(sum(o.sum() for o in ops.norm_rotate(*leaves, **more)), leaves), ops.norm_rotate_grad(*(t.detach() for t in leaves), *ones, **more)):
        assert torch.equal(x, y)


def test_streams_graphs_and_repeats(ops):
    q, k, _, gains, grads = inputs(3, 301, 8, 4, 128, BF16, seed=8)
    rope = ops.rope_table(301, 128)

    def run(*a):
        return [*ops.norm_rotate(*a[:4], rope=rope), *ops.norm_rotate_grad(*a, rope=rope)]
    want = run(q, k, *gains, *grads)
    q2, k2, _, gains2, grads2 = inputs(3, 301, 8, 4, 128, BF16, seed=9)
    want2 = run(q2, k2, *gains2, *grads2)
    static = [t.clone() for t in (q, k, *gains, *grads)]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        cap = run(*static)
    outs, sides = [], [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    for _ in range(10):
        for s in sides:
            with torch.cuda.stream(s):
                outs.append(run(q, k, *gains, *grads))
    graph.replay()
    torch.cuda.synchronize()
    for got in outs + [cap]:
        assert all(torch.equal(x, y) for x, y in zip(got, want))
    for a, b in zip(static, (q2, k2, *gains2, *grads2)):
        a.copy_(b)
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(cap, want2))


def test_offsets_beyond_32_bits(ops):
    """Rows more than 2^31 elements apart."""
    big = torch.empty(2 ** 31 + 10 * 4 * 64, dtype=BF16, device="cuda")
    q = torch.as_strided(big, (2, 10, 4, 64), (2 ** 31, 256, 64, 1))
    q.copy_(torch.randn((2, 10, 4, 64), device="cuda"))
    gain = torch.ones(64, device="cuda")
    rope = ops.rope_table(10, 64)
    out, _ = ops.norm_rotate(q, None, gain, None, rope=rope)
    near(out, *ref.norm(q, gain, rope, None, EPS, False), "q")


def test_refusals(ops):
    q, k, _, gains, grads = inputs(2, 5, 4, 2, 64, BF16)
    rope = ops.rope_table(5, 64)
    for bad in (dict(q=None), dict(q=None, k=None, q_gain=None, k_gain=None), dict(k_gain=None), dict(q_gain=gains[0][:32]), dict(q_gain=gains[0].half()), dict(q_gain=gains[0].cpu()),
                dict(q=q.cpu()), dict(k=k.cpu()), dict(q=q[0]), dict(k=k[:, :4]), dict(k=k.float()), dict(q=q.long()), dict(q=q[..., :48], k=k[..., :48], q_gain=gains[0][:48], k_gain=gains[1][:48]),
                dict(q=q.transpose(2, 3), k=k.transpose(2, 3)), dict(rope=rope.double()), dict(rope=rope.cpu()), dict(rope=rope[:, :, :1]), dict(rope=ops.rope_table(5, 128)),
                dict(rope=rope[:0]), dict(positions=torch.zeros((2, 5), dtype=torch.int64, device="cuda")), dict(positions=torch.zeros((2, 4), dtype=torch.int32, device="cuda")),
                dict(positions=torch.zeros((5, 2), dtype=torch.int32, device="cuda").T), dict(eps=-1.0), dict(eps=math.nan), dict(eps=math.inf), dict(eps=1e300), dict(interleaved=2 ** 40)):
        args = dict(q=q, k=k, q_gain=gains[0], k_gain=gains[1], rope=rope)
        args.update(bad)
        with pytest.raises((ValueError, RuntimeError)):
            ops.norm_rotate(**args)
        with pytest.raises((ValueError, RuntimeError)):
            ops.norm_rotate_grad(**args, grad_q=grads[0], grad_k=grads[1])
    for bad in (dict(grad_q=None), dict(grad_k=None), dict(grad_q=grads[0][:, :4]), dict(grad_q=grads[0].float()), dict(grad_k=grads[1].cpu())):
        args = dict(grad_q=grads[0], grad_k=grads[1])
        args.update(bad)
        with pytest.raises(ValueError):
            ops.norm_rotate_grad(q, k, *gains, **args, rope=rope)
    qg = q.clone().requires_grad_()
    with pytest.raises(ValueError, match="no_grad"):
        ops.norm_rotate_grad(qg, k, *gains, *grads, rope=rope)
    with pytest.raises(ValueError, match="rope"):
        ops.norm_rotate(q, k, *gains, rope=rope.clone().requires_grad_())
    (g1,) = torch.autograd.grad(ops.norm_rotate(qg, k, *gains, rope=rope)[0].float().sum(), qg, create_graph=True)
    with pytest.raises(RuntimeError):
        torch.autograd.grad(g1.float().sum(), qg)
    with torch.autograd.forward_ad.dual_level():
        with pytest.raises(ValueError, match="forward-mode"):
            ops.norm_rotate(torch.autograd.forward_ad.make_dual(q.clone(), q.clone()), k, *gains, rope=rope)


# --------------------------------------------------------------------------------------------------------- into a paged cache

def cache_of(ops, n_pages, kv_heads, page, d, dtype, layout, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    shape = (n_pages, kv_heads, page, d) if layout == "hnd" else (n_pages, page, kv_heads, d)
    pools = [torch.randn(shape, generator=g, device="cuda").to(dtype) for _ in range(2)]
    pools = pools if layout == "hnd" else [p.transpose(1, 2) for p in pools]
    return ops.PagedCache(*pools), *pools


def check_append(ops, in_t, cache_t, batch=3, m=7, heads=4, kv_heads=2, d=64, page=16, rot=64, interleaved=False, layout="hnd", counts=None, queries=True, bad_pages=False, seed=0):
    q, k, v, gains, _ = inputs(batch, m, heads, kv_heads, d, in_t, seed)
    rope = ops.rope_table(60 + m, rot) if rot else None
    starts = torch.randint(0, 50, (batch,), device="cuda", dtype=torch.int32)
    width = (60 + m) // page + 1
    n_pages = batch * width + 2
    table = torch.randperm(n_pages, device="cuda")[:batch * width].view(batch, width).to(torch.int32)
    if bad_pages:
        table[0, int(starts[0]) // page] = -1
        table[1, int(starts[1]) // page] = n_pages
        starts[2] = -3
    cache, kp, vp = cache_of(ops, n_pages, kv_heads, page, d, cache_t, layout, seed + 1)
    k0, v0 = kp.clone(), vp.clone()
    c = None if counts is None else torch.tensor(counts, dtype=torch.int32, device="cuda")
    out = cache.append(k, v, table, starts, counts=c, q=q if queries else None, rope=rope, interleaved=interleaved, q_gain=gains[0] if queries else None, k_gain=gains[1])
    pos = starts.long()[:, None] + torch.arange(m, device="cuda")
    real = torch.arange(m, device="cuda") < (torch.full((batch, 1), m, device="cuda") if c is None else c[:, None])
    at = torch.where(real, pos, -1).to(torch.int32)
    if queries:
        live = real
        want, bound = ref.norm(q, gains[0], rope, at, EPS, interleaved)
        near(out, torch.where(live[..., None, None], want, 0.0), torch.where(live[..., None, None], bound, 0.0), "q")
    else:
        assert out is None
    want, bound = ref.norm(k, gains[1], rope, at, EPS, interleaved, cache_t)
    if cache_t is F16:
        want = want.clamp(-65504, 65504)
    seen = torch.zeros(kp.shape[0], kp.shape[2], dtype=torch.bool, device="cuda")
    for b in range(batch):
        for j in range(m):
            p = int(pos[b, j])
            if not bool(real[b, j]) or p < 0:
                continue
            g = int(table[b, p // page])
            if not 0 <= g < n_pages:
                continue
            near(kp[g, :, p % page], want[b, j], bound[b, j], "k")
            near(vp[g, :, p % page], v[b, j].double().clamp(-65504, 65504) if cache_t is F16 else v[b, j].double(), ref.stored(v[b, j].double(), torch.zeros((), dtype=torch.float64, device="cuda"), cache_t), "v")
            seen[g, p % page] = True
    keep = ~seen[:, None, :, None].expand_as(kp)
    assert torch.equal(kp[keep], k0[keep]) and torch.equal(vp[keep], v0[keep])


@pytest.mark.parametrize("in_t,cache_t", [(F32, F32), (F32, F16), (F32, BF16), (BF16, BF16), (BF16, F16), (F16, F16), (F16, F32), (BF16, F32)])
@pytest.mark.parametrize("rot", [64, 6])
def test_append_types(ops, in_t, cache_t, rot):
    check_append(ops, in_t, cache_t, rot=rot)


@pytest.mark.parametrize("d,heads,kv_heads,page,rot,interleaved,layout", [(32, 4, 4, 16, 32, False, "hnd"), (96, 6, 3, 48, 48, True, "nhd"), (128, 16, 2, 64, 128, True, "hnd"), (256, 4, 1, 32, 0, False, "nhd")])
def test_append_layouts(ops, d, heads, kv_heads, page, rot, interleaved, layout):
    check_append(ops, BF16, F16, d=d, heads=heads, kv_heads=kv_heads, page=page, rot=rot, interleaved=interleaved, layout=layout, seed=2)


def test_append_counts_places_and_long_prompts(ops):
    check_append(ops, BF16, BF16, counts=[0, 3, 9], seed=3)
    check_append(ops, BF16, BF16, queries=False, seed=4)
    check_append(ops, F32, F16, bad_pages=True, seed=5)
    check_append(ops, BF16, F16, batch=2, m=400, heads=8, kv_heads=4, d=128, rot=128, seed=6)
    check_append(ops, BF16, F16, batch=1, m=1, seed=7)


def test_append_of_equal_heads_is_the_append_of_normed_ones(ops):
    """Norms of their own before an append without any, in fp32: the same but for the roundings between."""
    q, k, v, gains, _ = inputs(2, 5, 4, 4, 64, F32, seed=8)
    rope = ops.rope_table(40, 64)
    table = torch.arange(6, dtype=torch.int32, device="cuda").view(2, 3)
    starts = torch.tensor([3, 11], dtype=torch.int32, device="cuda")
    a, ka, va = cache_of(ops, 6, 4, 16, 64, F32, "hnd", 9)
    b, kb, vb = cache_of(ops, 6, 4, 16, 64, F32, "hnd", 9)
    x = a.append(k, v, table, starts, q=q, rope=rope, q_gain=gains[0], k_gain=gains[1])
    nq, nk = ops.norm_rotate(q, k, *gains)
    y = b.append(nk, v, table, starts, q=nq, rope=rope)
    near(x, y, y.double().abs() * 2.0 ** -20 + y.double().abs().amax(-1, keepdim=True) * 2.0 ** -20, "q")
    near(ka, kb, kb.double().abs().amax(-1, keepdim=True) * 2.0 ** -19, "k")
    assert torch.equal(va, vb)


def test_append_refusals(ops):
    q, k, v, gains, _ = inputs(2, 5, 4, 2, 64, BF16)
    cache, _, _ = cache_of(ops, 8, 2, 16, 64, BF16, "hnd", 0)
    table, starts = torch.zeros((2, 2), dtype=torch.int32, device="cuda"), torch.zeros(2, dtype=torch.int32, device="cuda")
    good = dict(q=q, q_gain=gains[0], k_gain=gains[1])
    for bad in (dict(q_gain=None), dict(k_gain=None), dict(q=None), dict(k_gain=gains[1][:32]), dict(q_gain=gains[0].half()), dict(k_gain=gains[1].cpu()), dict(eps=-1.0), dict(eps=math.nan),
                dict(eps=1e300), dict(k_gain=gains[1].clone().requires_grad_()), dict(rope=ops.rope_table(4, 64)[:0])):
        with pytest.raises((ValueError, RuntimeError)):
            cache.append(k, v, table, starts, **{**good, **bad})
