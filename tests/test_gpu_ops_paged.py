"""Appending to and attending over a caller's paged pools, against plain loops in 64 bits."""
import math

import pytest
import torch

import ops_reference as ref
from ops_reference import TINY, UNIT

pytestmark = pytest.mark.gpu

F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16


@pytest.fixture(scope="module")
def ops():
    assert torch.cuda.is_available(), "this test needs a B200"
    from paper_2507_23777_b200 import build, ops
    build.build()
    return ops


def gen(seed):
    return torch.Generator().manual_seed(seed)


def where(x, layout):
    """To the GPU, a pool laid out [pages, page_size, heads, d] as the view of one that is."""
    return x.transpose(1, 2).contiguous().cuda().transpose(1, 2) if layout == "nhd" else x.contiguous().cuda()


def close(got, want, bound, what):
    got = got.detach().cpu().double()
    assert torch.equal(torch.isfinite(got), torch.isfinite(want)), what
    fine = torch.isfinite(want)
    assert torch.equal(got[~fine].nan_to_num(7.0), want[~fine].nan_to_num(7.0)), what
    off = (got - want).abs()[fine]
    over = off > bound.expand_as(want)[fine]
    assert not over.any(), f"{what}: {int(over.sum())} of {over.numel()} beyond the bound, worst {float((off / bound.expand_as(want)[fine]).max()):.3g} of it"


def check_attend(ops, cache_t, q_t, d, hk, group, m, page, lens, causal=True, window=0, layout="hnd", counts=None, fill=math.nan, scale=None,
                 seed=0, spread=2.0, break_table=None):
    g = gen(seed)
    k, v, table = ref.pools(g, lens, hk, page, d, cache_t, layout, fill=fill)
    if break_table is not None:
        break_table(table, k.shape[0])
    q = (spread * torch.randn((len(lens), m, hk * group, d), generator=g)).to(q_t)
    want, lse, weight, score = ref.attend(q, k, v, table, lens, counts, causal, window, scale)
    cache = ops.PagedCache(where(k, layout), where(v, layout))
    ints = lambda x: None if x is None else torch.tensor(x, dtype=torch.int32, device="cuda")
    got, got_lse = cache.attend(q.cuda(), table.cuda(), ints(lens), counts=ints(counts), causal=causal, window=window, scale=scale)
    # Scores: products of d elements, 2^-21 of the terms' size (the fp32 ones as three products of parts of eleven bits), queries split
    # over a 16-bit pool 2^-22.  Weights: that much times the score, and their own rounding, 2^-11 where the output has no more bits
    # than the weights, else 2^-16; every sum of n terms n 2^-24.
    n = max(1, max(lens, default=1))
    s = (2.0 ** -21 + d * 2.0 ** -24) * score + 2.0 ** -22
    rounding = 2.0 ** -20 if cache_t is F32 else 2.0 ** -11 if (cache_t, q_t) == (F16, BF16) else 2.0 ** -16
    close(got, want, UNIT[q_t] * want.abs() + (2 * s[..., None] + rounding + n * 2.0 ** -24) * weight + TINY[q_t], "out")
    close(got_lse, lse, 2.0 ** -22 * lse.abs().nan_to_num(posinf=1.0) + s + n * 2.0 ** -24, "lse")
    return got


TYPES = [(F16, F16), (F16, BF16), (F16, F32), (BF16, BF16), (F32, F32)]


@pytest.mark.parametrize("cache_t,q_t", TYPES)
@pytest.mark.parametrize("d", [32, 64, 96, 128, 256])
def test_attend_types_and_widths(ops, cache_t, q_t, d):
    """Ragged lengths on both sides of pages and of every tile: none, one, a page, one more, several hundred."""
    check_attend(ops, cache_t, q_t, d, 2, 2, 3, 16, [0, 1, 2, 16, 17, 31, 33, 200, 391], seed=d)


@pytest.mark.parametrize("cache_t,q_t", TYPES)
@pytest.mark.parametrize("hk,group,m", [(1, 1, 1), (3, 1, 16), (1, 7, 1), (2, 5, 4), (1, 8, 16), (2, 16, 2), (1, 71, 1), (4, 3, 5)])
def test_attend_head_layouts_and_windows_of_tokens(ops, cache_t, q_t, hk, group, m):
    """One row to 128 rows that share a key head."""
    check_attend(ops, cache_t, q_t, 64, hk, group, m, 32, [5, 70, 333], seed=hk * group + m)


@pytest.mark.parametrize("cache_t,q_t", TYPES)
@pytest.mark.parametrize("page", [16, 32, 48, 64, 112, 128])
def test_attend_pages_and_pool_layouts(ops, cache_t, q_t, page):
    for layout in ("hnd", "nhd"):
        check_attend(ops, cache_t, q_t, 64, 3, 1, 2, page, [page - 1, page, page + 1, 3 * page + 5], layout=layout, seed=page)


@pytest.mark.parametrize("cache_t,q_t", TYPES)
@pytest.mark.parametrize("window", [1, 2, 15, 16, 17, 64, 100, 1000])
def test_attend_sliding_window(ops, cache_t, q_t, window):
    """Keys before the window hold NaN in no case, but what they hold must not matter."""
    check_attend(ops, cache_t, q_t, 64, 2, 2, 4, 32, [3, 65, 230, 400], window=window, seed=window)


@pytest.mark.parametrize("cache_t,q_t", TYPES)
def test_attend_without_causal_order_and_with_counts(ops, cache_t, q_t):
    check_attend(ops, cache_t, q_t, 64, 2, 1, 5, 64, [257, 1, 0, 64], causal=False, seed=1)
    check_attend(ops, cache_t, q_t, 64, 2, 2, 5, 64, [257, 3, 0, 64, 40], counts=[5, 5, 2, 0, 1], seed=2)
    check_attend(ops, cache_t, q_t, 64, 2, 2, 5, 64, [257, 3, 70], counts=[4, 1, 3], causal=False, seed=3)


@pytest.mark.parametrize("cache_t,q_t", TYPES)
@pytest.mark.parametrize("lens", [[3000], [5000, 1], [1200] * 40, [0] * 30 + [2500], [700 * (i % 5) + i for i in range(33)]])
def test_attend_split_over_the_length(ops, cache_t, q_t, lens):
    """Few sequences whose keys are cut over the chip, and many that are cut here and there."""
    check_attend(ops, cache_t, q_t, 32, 1, 1, 1, 64, lens, seed=len(lens))


def test_attend_many_key_heads(ops):
    check_attend(ops, BF16, BF16, 32, 200, 1, 1, 16, [40, 90], seed=5)


@pytest.mark.parametrize("cache_t,q_t", TYPES)
@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf])
def test_attend_is_blind_to_what_a_row_does_not_see(ops, cache_t, q_t, bad):
    """A key or value that only later rows of a window see, or that lies before a row's sliding window, is anything: the rows that do not see it
    are exact."""
    d, m, lens, page = 64, 4, [37, 97, 260], 32
    for window in (0, 6, 40):
        g = gen(int(window))
        k, v, table = ref.pools(g, lens, 1, page, d, cache_t, fill=bad)
        q = torch.randn((3, m, 2, d), generator=g).to(q_t)
        want, _, weight, score = ref.attend(q, k, v, table, lens, None, True, window)
        for victim in ("k", "v"):
            kk, vv = k.clone(), v.clone()
            for b, n in enumerate(lens):
                for p in [n - 1, n - 2] + ([n - m - window] if window and n - m - window >= 0 else []):
                    (kk if victim == "k" else vv)[table[b, p // page], 0, p % page, ::3] = bad
            cache = ops.PagedCache(kk.cuda(), vv.cuda())
            got, lse = cache.attend(q.cuda(), table.cuda(), torch.tensor(lens, dtype=torch.int32, device="cuda"), window=window)
            # rows 0 and 1 see positions up to n - 4 and n - 3: neither of the two newest
            s = (2.0 ** -21 + d * 2.0 ** -24) * score + 2.0 ** -22
            bound = UNIT[q_t] * want.abs() + (2 * s[..., None] + 2.0 ** -11 + 260 * 2.0 ** -24) * weight + TINY[q_t]
            close(got[:, :2], want[:, :2], bound[:, :2], f"{victim} {window}")
            if victim == "v":      # and a row that sees it has it
                assert not torch.isfinite(got[:, 3, :, 0]).any()
                assert torch.isfinite(got[:, 3, :, 1]).all() and torch.isfinite(lse).all()


@pytest.mark.parametrize("cache_t,q_t", TYPES)
def test_attend_ignores_pages_outside_the_pool(ops, cache_t, q_t):
    def broken(table, n):
        table[0, 0], table[0, 2], table[1, 1], table[2, :] = -1, n, 2 ** 31 - 1, -5
    check_attend(ops, cache_t, q_t, 64, 2, 1, 2, 32, [150, 90, 40], seed=4, break_table=broken)


def test_attend_lengths_beyond_the_table_end_there(ops):
    g = gen(3)
    k, v, table = ref.pools(g, [64], 1, 32, 64, F16)
    table = table[:, :2]
    q = torch.randn((1, 2, 1, 64), generator=g).to(F16)
    cache = ops.PagedCache(k.cuda(), v.cuda())
    a = cache.attend(q.cuda(), table.cuda(), torch.tensor([64], dtype=torch.int32, device="cuda"))
    b = cache.attend(q.cuda(), table.cuda(), torch.tensor([2 ** 31 - 1], dtype=torch.int32, device="cuda"))
    c = cache.attend(q.cuda(), table.cuda(), torch.tensor([-7], dtype=torch.int32, device="cuda"))
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
    assert not c[0].any() and (c[1] == -math.inf).all()


@pytest.mark.parametrize("cache_t,q_t", TYPES)
def test_attend_large_scores_and_scales(ops, cache_t, q_t):
    """Softmax of scores in the hundreds (one key has it all), a scale of zero (all alike) and a negative one."""
    for scale in (3.0, 0.0, -0.2):
        check_attend(ops, cache_t, q_t, 64, 1, 2, 2, 32, [100, 45], scale=scale, seed=6)


def test_attend_strides_and_out(ops):
    """Queries out of a joint projection, output into a larger buffer, table with a row stride of its own."""
    g = gen(9)
    lens = [130, 77]
    k, v, table = ref.pools(g, lens, 2, 32, 64, BF16)
    qkv = torch.randn((2, 3, 8, 64), generator=g).to(BF16).cuda()
    q = qkv[:, :, 1:5]
    wide = torch.full((2, table.shape[1] + 3), 7, dtype=torch.int32)
    wide[:, :table.shape[1]] = table
    cache = ops.PagedCache(k.cuda(), v.cuda())
    n = torch.tensor(lens, dtype=torch.int32, device="cuda")
    want, lse = cache.attend(q.contiguous(), table.cuda(), n)
    buf = torch.full((3, 2, 6, 64), 5.0, dtype=BF16, device="cuda")
    out = buf.transpose(0, 1)[:, :, 1:5]
    got, lse2 = cache.attend(q, wide.cuda()[:, :table.shape[1]], n, out=out)
    assert got is out and torch.equal(got, want) and torch.equal(lse, lse2)
    assert (buf[:, :, 0] == 5).all() and (buf[:, :, 5] == 5).all()


def test_attend_repeats_bit_for_bit_on_streams_and_in_a_graph(ops):
    """The same call again, on other streams at the same time, and replayed: bit for bit the same."""
    g = gen(10)
    lens = [4000, 10, 2500, 900]
    k, v, table = ref.pools(g, lens, 2, 64, 64, F16)
    q = torch.randn((4, 5, 4, 64), generator=g).to(F16).cuda()
    cache = ops.PagedCache(k.cuda(), v.cuda())
    table, n = table.cuda(), torch.tensor(lens, dtype=torch.int32, device="cuda")
    want, lse = cache.attend(q, table, n)
    for _ in range(20):
        got, l2 = cache.attend(q, table, n)
        assert torch.equal(got, want) and torch.equal(l2, lse)
    streams = [torch.cuda.Stream() for _ in range(3)]
    torch.cuda.synchronize()
    outs = []
    for _ in range(10):
        for s in streams:
            with torch.cuda.stream(s):
                outs.append(cache.attend(q, table, n))
    torch.cuda.synchronize()
    assert all(torch.equal(o, want) and torch.equal(l2, lse) for o, l2 in outs)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out, l2 = cache.attend(q, table, n)
    for _ in range(3):
        out.zero_(), l2.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want) and torch.equal(l2, lse)


def test_graph_keeps_its_workspace(ops):
    """A graph, then a call on the same stream that wants a larger workspace: the graph's is not handed out again."""
    g = gen(31)
    lens = [4000, 10, 2500, 900]
    k, v, table = ref.pools(g, lens, 2, 64, 64, F16)
    q = torch.randn((4, 16, 8, 64), generator=g).to(F16).cuda()
    few = q[:, :1, :4].contiguous()
    cache = ops.PagedCache(k.cuda(), v.cuda())
    table, n = table.cuda(), torch.tensor(lens, dtype=torch.int32, device="cuda")
    stream = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(stream):
        want, _ = cache.attend(few, table, n)
        small = cache._ws[stream.cuda_stream][0]
        at, size = small.data_ptr(), small.numel()
        del small
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=stream):
        out, _ = cache.attend(few, table, n)
    with torch.cuda.stream(stream):
        cache.attend(q, table, n)
        assert cache._ws[stream.cuda_stream][1] > size
        others = [torch.full((size,), 85, dtype=torch.uint8, device="cuda") for _ in range(4)]
        assert all(not o.data_ptr() <= at < o.data_ptr() + o.numel() for o in others)
        graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(out, want) and all((o == 85).all() for o in others)
    cache.check()


def test_attend_offsets_beyond_32_bits(ops):
    """A pool of more than 2^32 elements: the pages at its end."""
    n_pages, page, d = 1100, 4096 * 4, 256
    pool = torch.zeros((2, n_pages, 1, page, d), dtype=BF16, device="cuda")
    g = gen(12)
    rows = torch.randn((2, 20, d), generator=g).to(BF16)
    pool[:, n_pages - 1, 0, :20] = rows.cuda()
    cache = ops.PagedCache(pool[0], pool[1])
    assert pool[0].numel() > 2 ** 32
    q = torch.randn((1, 1, 1, d), generator=g).to(BF16)
    table = torch.tensor([[n_pages - 1]], dtype=torch.int32, device="cuda")
    got, _ = cache.attend(q.cuda(), table, torch.tensor([20], dtype=torch.int32, device="cuda"))
    s = torch.softmax(d ** -0.5 * (rows[0].double() @ q[0, 0, 0].double()), 0) @ rows[1].double()
    assert float((got[0, 0, 0].cpu().double() - s).norm() / s.norm()) < 2.0 ** -8
    new = torch.ones((1, 1, 1, d), dtype=BF16, device="cuda")
    cache.append(2 * new, 3 * new, table, torch.tensor([page - 1], dtype=torch.int32, device="cuda"))
    assert (pool[0, -1, 0, -1] == 2).all() and (pool[1, -1, 0, -1] == 3).all()
    assert int(torch.count_nonzero(pool[0])) == d + int(torch.count_nonzero(rows[0]))


def check_append(ops, cache_t, in_t, d, hk, heads, m, page, starts, rot=None, interleaved=False, counts=None, layout="hnd", seed=0,
                 break_table=None, positions=None, packed=True, magnitude=1.0):
    g = gen(seed)
    batch = len(starts)
    kp, vp, table = ref.pools(g, [max(0, s) + m for s in starts], hk, page, d, cache_t, layout)
    if break_table is not None:
        break_table(table, kp.shape[0])
    x = (magnitude * torch.randn((batch, m, heads + 2 * hk, d), generator=g)).to(in_t)
    gx = x.cuda()
    q, k, v = x.split([heads, hk, hk], 2)
    gq, gk, gv = gx.split([heads, hk, hk], 2)
    if not packed:
        gq, gk, gv = gq.contiguous(), gk.contiguous(), gv.contiguous()
    rope = None if rot is None else ops.rope_table(positions or max(starts) + m, rot)
    ints = lambda t: None if t is None else torch.tensor(t, dtype=torch.int32, device="cuda")
    gk_pool, gv_pool = where(kp, layout), where(vp, layout)
    cache = ops.PagedCache(gk_pool, gv_pool)
    out = cache.append(gk, gv, table.cuda(), ints(starts), counts=ints(counts), q=gq if heads else None, rope=rope, interleaved=interleaved)
    q_out, want_k, want_v, q_w, k_w = ref.append(q if heads else None, k, v, kp, vp, table, starts, counts, None if rope is None else rope.cpu(), interleaved)
    # two products and a sum in fp32, 2^-22 of the two elements' size, then one rounding
    if heads:
        close(out, q_out, UNIT[in_t] * q_out.abs() + 2.0 ** -22 * q_w + TINY[in_t], "q")
    else:
        assert out is None
    if cache_t is F16:
        want_k, want_v = want_k.clamp(-65504, 65504), want_v.clamp(-65504, 65504)
    changed = k_w > 0
    bound_k = torch.where(changed, UNIT[cache_t] * want_k.abs() + 2.0 ** -22 * k_w + TINY[cache_t], 0.0)
    close(gk_pool, want_k, bound_k, "keys")
    exact_v = want_v.to(torch.float32).to(cache_t).double()      # one rounding of what was given
    assert torch.equal(gv_pool.cpu().double(), exact_v), "values"


@pytest.mark.parametrize("cache_t", [F32, BF16, F16])
@pytest.mark.parametrize("in_t", [F32, BF16, F16])
def test_append_types(ops, cache_t, in_t):
    for d in (32, 64, 96, 128, 256):
        check_append(ops, cache_t, in_t, d, 2, 4, 3, 32, [0, 31, 100], rot=d, seed=d)


@pytest.mark.parametrize("rot,interleaved", [(None, False), (2, False), (2, True), (10, False), (10, True), (16, False), (16, True), (32, True), (48, False), (64, True), (64, False)])
def test_append_rotations(ops, rot, interleaved):
    """Whole heads and parts of them, in pieces of sixteen elements and not; both pairings."""
    check_append(ops, F16, BF16, 64, 3, 3, 4, 16, [0, 13, 500], rot=rot, interleaved=interleaved, seed=2)
    check_append(ops, F32, F32, 64, 1, 5, 4, 16, [7, 90], rot=rot, interleaved=interleaved, seed=3, packed=False)


@pytest.mark.parametrize("layout", ["hnd", "nhd"])
def test_append_layouts_counts_and_long_prompts(ops, layout):
    check_append(ops, BF16, BF16, 64, 2, 0, 1, 48, [47, 48, 0, 95], rot=64, layout=layout, seed=4)
    check_append(ops, F16, F32, 64, 2, 2, 70, 16, [0, 5, 9], rot=32, counts=[70, 0, 33], layout=layout, seed=5)
    check_append(ops, BF16, BF16, 32, 1, 1, 1500, 64, [3], rot=32, layout=layout, seed=6)


def test_append_leaves_out_tokens_without_a_place(ops):
    """Negative positions, positions beyond the table and the rope, page numbers outside the pool."""
    def broken(table, n):
        table[0, 0], table[1, 0] = -1, n
    check_append(ops, F16, F16, 64, 2, 2, 40, 16, [0, 0, -20], rot=64, seed=7, break_table=broken)
    check_append(ops, F16, F16, 64, 2, 2, 40, 16, [0, 90], rot=64, positions=100, seed=8)
    check_append(ops, F16, F16, 64, 2, 2, 40, 16, [-20, -40], seed=9)


def test_append_saturates_fp16_and_keeps_nan(ops):
    check_append(ops, F16, F32, 64, 2, 2, 4, 16, [5], rot=64, magnitude=1e5, seed=10)
    kp = torch.zeros((1, 1, 16, 64), dtype=F16, device="cuda")
    cache = ops.PagedCache(kp, kp.clone())
    x = torch.full((1, 1, 1, 64), math.nan, device="cuda")
    cache.append(x, x * math.inf, torch.zeros((1, 1), dtype=torch.int32, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda"))
    assert kp[0, 0, 0].isnan().all() and cache.v[0, 0, 0].isnan().all() and not kp[0, 0, 1:].any()


def test_append_in_place_and_empty_calls(ops):
    g = gen(11)
    kp = torch.randn((4, 2, 16, 64), generator=g).to(BF16).cuda()
    cache = ops.PagedCache(kp, kp.clone())
    q = torch.randn((1, 3, 2, 64), generator=g).to(BF16).cuda()
    k = torch.randn((1, 3, 2, 64), generator=g).to(BF16).cuda()
    table, starts = torch.tensor([[2, 0]], dtype=torch.int32, device="cuda"), torch.tensor([14], dtype=torch.int32, device="cuda")
    rope = ops.rope_table(32, 64)
    want = cache.append(k, k, table, starts, q=q, rope=rope)
    mine = q.clone()
    assert cache.append(k, k, table, starts, q=mine, rope=rope, out=mine) is mine and torch.equal(mine, want)
    before = kp.clone()
    cache.append(k[:, :0], k[:, :0], table, starts)
    cache.append(k[:0], k[:0], table[:0], starts[:0])
    out, lse = cache.attend(q[:0], table[:0], starts[:0])
    assert torch.equal(kp, before) and out.shape == (0, 3, 2, 64) and lse.shape == (0, 3, 2)


def test_append_then_attend_equals_attention_over_whole_sequences(ops):
    """Three windows appended and attended one after the other = causal attention over the rotated sequence."""
    g = gen(13)
    h, d, steps, m = 4, 64, 5, 7
    kp, vp = (torch.zeros((8, h, 16, d), dtype=F32, device="cuda") for _ in range(2))
    cache = ops.PagedCache(kp, vp)
    table = torch.tensor([[3, 1, 6]], dtype=torch.int32, device="cuda")
    x = torch.randn((3, 1, steps * m, h, d), generator=g)
    rope = ops.rope_table(steps * m, d)
    rows = []
    for s in range(steps):
        q, k, v = (t[:, s * m:(s + 1) * m].cuda() for t in x)
        start = torch.tensor([s * m], dtype=torch.int32, device="cuda")
        rows.append(cache.attend(cache.append(k, v, table, start, q=q, rope=rope), table, start + m)[0])
    got = torch.cat(rows, 1).cpu().double()

    def turned(t):
        c, s = rope.cpu().double().unbind(-1)
        a, b = t[0].double().split(d // 2, -1)
        c, s = c[:, None], s[:, None]
        return torch.cat([a * c - b * s, a * s + b * c], -1)
    q, k = turned(x[0]), turned(x[1])
    s = torch.einsum("ihd,jhd->hij", q, k) / d ** 0.5
    s = s.masked_fill(torch.ones(steps * m, steps * m, dtype=torch.bool).triu(1), -math.inf)
    want = torch.einsum("hij,jhd->ihd", torch.softmax(s, -1), x[2][0].double())
    assert float((got[0] - want).norm() / want.norm()) < 2.0 ** -19


def test_refusals(ops):
    from paper_2507_23777_b200.binding import XsmError
    kp = torch.zeros((4, 2, 32, 64), dtype=F16, device="cuda")
    cache = ops.PagedCache(kp, kp.clone())
    table, one = torch.zeros((1, 4), dtype=torch.int32, device="cuda"), torch.ones(1, dtype=torch.int32, device="cuda")
    q = torch.zeros((1, 1, 2, 64), dtype=F16, device="cuda")
    both = (ValueError, XsmError)
    for make in (lambda: ops.PagedCache(kp[:, :, :24], kp[:, :, :24]), lambda: ops.PagedCache(kp[..., :48], kp[..., :48]), lambda: ops.PagedCache(kp, kp.float()),
                 lambda: ops.PagedCache(kp.cpu(), kp.cpu()), lambda: ops.PagedCache(kp.long(), kp.long()), lambda: ops.PagedCache(kp[..., ::2], kp[..., ::2]),
                 lambda: ops.PagedCache(kp.flatten()[4:4 + 64 * 32].view(1, 1, 32, 64), kp.flatten()[4:4 + 64 * 32].view(1, 1, 32, 64))):
        with pytest.raises(both):
            make()
    for call in (lambda: cache.attend(q[0], table, one), lambda: cache.attend(q.repeat(1, 17, 1, 1), table, one), lambda: cache.attend(q[..., :32], table, one),
                 lambda: cache.attend(q.repeat(1, 1, 2, 1)[:, :, :3], table, one), lambda: cache.attend(q, table.long(), one), lambda: cache.attend(q, table, one.long()),
                 lambda: cache.attend(q, table.repeat(2, 1), one), lambda: cache.attend(q, table, one.repeat(2)), lambda: cache.attend(q, table, one, window=-1),
                 lambda: cache.attend(q, table, one, window=3, causal=False), lambda: cache.attend(q, table, one, scale=math.nan),
                 lambda: cache.attend(q.cpu(), table, one), lambda: cache.attend(q, table.cpu(), one), lambda: cache.attend(q, table, one, out=q.float()),
                 lambda: cache.attend(q.clone().requires_grad_(), table, one), lambda: cache.attend(q, table, one, lse=torch.empty(1, device="cuda")),
                 lambda: cache.attend(torch.zeros((1, 1, 2, 68), dtype=F16, device="cuda")[..., 1:65], table, one),
                 lambda: cache.append(q, q[:, :, :1], table, one), lambda: cache.append(q, q.float(), table, one), lambda: cache.append(q, q, table, one, q=q.float()),
                 lambda: cache.append(q, q, table, one, rope=torch.zeros((4, 33, 2), device="cuda")), lambda: cache.append(q, q, table, one, rope=torch.zeros((4, 32, 2), dtype=F16, device="cuda")),
                 lambda: cache.append(q, q, table, one, counts=one.float()), lambda: cache.append(q, q, table, one, q=q, out=q[..., :32])):
        with pytest.raises(both):
            call()
    bf = ops.PagedCache(kp.to(BF16), kp.to(BF16))
    with pytest.raises(XsmError) as e:
        bf.attend(q, table, one)
    assert "q_dtype" in str(e.value)
    out, _ = cache.attend(q, table, one)          # and the cache is still good
    assert not out.any()


def test_a_wait_that_ran_out_is_told(ops):
    """The status word of a workspace, as a kernel would leave it."""
    from paper_2507_23777_b200.binding import XSM_ERR_TIMEOUT, XsmError
    kp = torch.zeros((4, 2, 32, 64), dtype=F16, device="cuda")
    cache = ops.PagedCache(kp, kp.clone())
    cache.check()
    q, table, one = torch.zeros((1, 1, 2, 64), dtype=F16, device="cuda"), torch.zeros((1, 4), dtype=torch.int32, device="cuda"), torch.ones(1, dtype=torch.int32, device="cuda")
    cache.attend(q, table, one)
    cache.check()
    (ws, _), = cache._ws.values()
    ws[:4].view(torch.int32)[0] = XSM_ERR_TIMEOUT
    with pytest.raises(XsmError) as e:
        cache.check()
    assert e.value.status == XSM_ERR_TIMEOUT
    cache.check()


@pytest.mark.parametrize("cache_t,q_t", TYPES)
@pytest.mark.parametrize("d,m,group", [(256, 5, 7), (128, 16, 3), (96, 16, 4), (256, 1, 1), (128, 1, 1), (64, 3, 11)])
def test_attend_wide_heads_with_many_rows_and_sliding_windows(ops, cache_t, q_t, d, m, group):
    """Warps that share a stage, row tiles in groups, masked stages in each."""
    for window in (0, 37):
        check_attend(ops, cache_t, q_t, d, 1, group, m, 48, [m + 1, 300, 129], window=window, seed=d + m)


@pytest.mark.parametrize("cache_t,q_t", TYPES)
def test_attend_exactness(ops, cache_t, q_t):
    """2-norm of the error against the norm of the result over 2500 keys: rounding to the output's type, 2^-9 and 2^-12 on average for numbers of eight
    and eleven bits; fp32 outputs 2^-20, a few roundings of the scores (of a size of eight and more) and of the sums."""
    g = gen(21)
    k, v, table = ref.pools(g, [2500], 2, 64, 64, cache_t)
    q = (2 * torch.randn((1, 3, 4, 64), generator=g)).to(q_t)
    want = ref.attend(q, k, v, table, [2500])[0]
    got, _ = ops.PagedCache(k.cuda(), v.cuda()).attend(q.cuda(), table.cuda(), torch.tensor([2500], dtype=torch.int32, device="cuda"))
    off = float((got.cpu().double() - want).norm() / want.norm())
    assert off < {F32: 2.0 ** -19, BF16: 2.0 ** -9, F16: 2.0 ** -12}[q_t], off


def test_attend_of_bf16_queries_over_fp16_pages_is_rounded_once(ops):
    """Against the 64-bit result rounded to bf16.  What is off by e (relative) before the rounding ends on the other side of a rounding's edge
    in about one of 2^-8 / e numbers, which is then off by up to 2^-8: sqrt(2^8 e) 2^-8 in norm.  Scores and weights of 22 bits and more
    leave e below 2^-18, 2^-13 in norm; weights of eleven bits 2^-13 over so many keys, 2^-10.5."""
    g = gen(22)
    k, v, table = ref.pools(g, [2500], 2, 64, 64, F16)
    q = (2 * torch.randn((1, 5, 4, 64), generator=g)).to(BF16)
    want = ref.attend(q, k, v, table, [2500])[0].float().to(BF16).double()
    got, _ = ops.PagedCache(k.cuda(), v.cuda()).attend(q.cuda(), table.cuda(), torch.tensor([2500], dtype=torch.int32, device="cuda"))
    off = float((got.cpu().double() - want).norm() / want.norm())
    assert off < 2.0 ** -12, off


@pytest.mark.parametrize("cache_t,q_t", TYPES)
@pytest.mark.parametrize("d,lens,m", [(64, [4000, 10, 0, 900], 5), (256, [300], 16), (128, [40] * 200, 1)])
def test_waits_that_run_out(ops, cache_t, q_t, d, lens, m):
    """Keys that are never fetched: after a few tries every wait gives up, the call ends, its status is told once, and the next call (on counters
    that have to be back at zero) is right."""
    from paper_2507_23777_b200.binding import XSM_ERR_TIMEOUT, XsmError
    g = gen(d)
    k, v, table = ref.pools(g, lens, 2, 32, d, cache_t)
    q = torch.randn((len(lens), m, 4, d), generator=g).to(q_t).cuda()
    cache, table, n = ops.PagedCache(k.cuda(), v.cuda()), table.cuda(), torch.tensor(lens, dtype=torch.int32, device="cuda")
    want, lse = cache.attend(q, table, n)
    cache.check()
    cache.lib.xsm_debug_kv_waits(cache._h, 20, 1)
    cache.attend(q, table, n)
    cache.lib.xsm_debug_kv_waits(cache._h, 0, 0)
    with pytest.raises(XsmError) as e:
        cache.check()
    assert e.value.status == XSM_ERR_TIMEOUT
    cache.check()
    got, lse2 = cache.attend(q, table, n)
    cache.check()
    assert torch.equal(got, want) and torch.equal(lse, lse2)


@pytest.mark.parametrize("cache_t,q_t", TYPES)
@pytest.mark.parametrize("nats", [8.0, 11.0, 15.0, 17.5, 18.0])
def test_attend_keys_far_below_one_without_a_value(ops, cache_t, q_t, nats):
    """A key that takes nearly all of the softmax and whose value is zero: what the others have is the whole result.  Over 16-bit pages a
    weight enters as two parts of the type, over fp16 ones of which 2^-24 is the smallest step and 2^15 the largest weight's size."""
    for n, at in ((201, 0), (201, 130), (201, 200), (2600, 5), (2600, 2599)):
        g = gen(n + at)
        k, v, table = ref.pools(g, [n], 1, 32, 64, cache_t)
        k.zero_()
        v.copy_(1 + torch.rand(v.shape, generator=g))
        k[table[0, at // 32], 0, at % 32, 0] = nats
        v[table[0, at // 32], 0, at % 32] = 0
        q = torch.zeros((1, 1, 2, 64), dtype=q_t)
        q[..., 0] = 1
        want, lse, _, _ = ref.attend(q, k, v, table, [n], scale=1.0)
        cache = ops.PagedCache(k.cuda(), v.cuda())
        got, got_lse = cache.attend(q.cuda(), table.cuda(), torch.tensor([n], dtype=torch.int32, device="cuda"), scale=1.0)
        part = {F16: max(2.0 ** -22, 2.0 ** -25 / (2.0 ** 15 * math.exp(-nats))), BF16: 2.0 ** -16, F32: 2.0 ** -20}[cache_t]
        # the exponent of 26 at most, its rounding 2^-24 of it; exponentials 2^-22; sums
        close(got, want, (UNIT[q_t] + part + 2.0 ** -18 + n * 2.0 ** -24) * want.abs() + TINY[q_t], "out")
        close(got_lse, lse, 2.0 ** -22 * lse.abs() + n * 2.0 ** -24, "lse")


@pytest.mark.parametrize("q_t", [F16, BF16, F32])
@pytest.mark.parametrize("scale", [2.0 ** e for e in range(0, 101, 5)])
def test_attend_scores_of_any_size_over_fp16_pages(ops, q_t, scale):
    """The largest score's weight is far from the largest fp16 number, and the reference that it is taken against is a rounded one: two equal
    keys above all others share the softmax evenly, whatever their score."""
    g = gen(1)
    k, v, table = ref.pools(g, [90], 1, 32, 64, F16)
    k.zero_()
    for at in (3, 77):
        k[table[0, at // 32], 0, at % 32, 0] = 1023.0
    q = torch.zeros((1, 1, 1, 64), dtype=q_t)
    q[..., 0] = 1
    cache = ops.PagedCache(k.cuda(), v.cuda())
    got, lse = cache.attend(q.cuda(), table.cuda(), torch.tensor([90], dtype=torch.int32, device="cuda"), scale=scale)
    a, b = (v[table[0, at // 32], 0, at % 32].double() for at in (3, 77))
    close(got[0, 0, 0], (a + b) / 2, UNIT[q_t] * ((a + b) / 2).abs() + 2.0 ** -20 * (a.abs() + b.abs()) + TINY[q_t], "out")
    close(lse[0, 0, 0], torch.tensor(1023.0 * scale + math.log(2.0), dtype=torch.float64), torch.tensor(1023.0 * scale * 2.0 ** -22 + 2.0 ** -20), "lse")


@pytest.mark.parametrize("cache_t,q_t", TYPES)
@pytest.mark.parametrize("window", [2 ** 31 - 1, 2 ** 31 - 2, 2 ** 31 - 10, 2 ** 31 - 40])
def test_attend_window_at_the_end_of_its_type(ops, cache_t, q_t, window):
    """A window that nothing lies before, over lengths below the number of new tokens too."""
    check_attend(ops, cache_t, q_t, 64, 2, 2, 5, 32, [1, 2, 3, 0, 40], window=window, seed=3)
    check_attend(ops, cache_t, q_t, 64, 1, 1, 16, 16, [1, 9, 16, 17], window=window, seed=4)
    check_attend(ops, cache_t, q_t, 32, 1, 1, 16, 64, [2000, 3], window=window, counts=[16, 12], seed=5)


def test_a_table_without_pages(ops):
    """Nothing has a place: nothing is written, nothing is seen, queries are rotated as ever."""
    g = gen(14)
    kp = torch.randn((4, 2, 16, 64), generator=g).to(F16).cuda()
    cache = ops.PagedCache(kp, kp.clone())
    before = kp.clone()
    x = torch.randn((3, 2, 2, 64), generator=g).to(F16).cuda()
    table, some, n = torch.zeros((3, 0), dtype=torch.int32, device="cuda"), torch.zeros((3, 1), dtype=torch.int32, device="cuda"), torch.tensor([0, 2, 9], dtype=torch.int32, device="cuda")
    rope = ops.rope_table(32, 64)
    q = cache.append(x, x, table, n, q=x, rope=rope)
    out, lse = cache.attend(x, table, n)
    assert torch.equal(kp, before) and torch.equal(cache.v, before)
    assert not out.any() and (lse == -math.inf).all()
    assert torch.equal(q, cache.append(x, x, some, n, q=x, rope=rope))


@pytest.mark.parametrize("cache_t,q_t", TYPES)
@pytest.mark.parametrize("sign", [1, -1])
def test_attend_largest_numbers_of_the_type(ops, cache_t, q_t, sign):
    """Keys and values of the type's largest and lowest number: rows that do not see them are exact, a row that sees nothing else has them."""
    d, m, n, page = 64, 4, 97, 32
    bad = sign * torch.finfo(cache_t).max
    g = gen(17)
    k, v, table = ref.pools(g, [n, 1], 1, page, d, cache_t, fill=bad)
    q = torch.randn((2, m, 2, d), generator=g).to(q_t)
    want, _, weight, score = ref.attend(q, k, v, table, [n, 1])
    s = (2.0 ** -21 + d * 2.0 ** -24) * score + 2.0 ** -22
    bound = UNIT[q_t] * want.abs() + (2 * s[..., None] + 2.0 ** -11 + 100 * 2.0 ** -24) * weight + TINY[q_t]
    for victim in (k, v):
        kept = victim.clone()
        for p in (n - 1, n - 2):
            victim[table[0, p // page], 0, p % page, ::3] = bad
        victim[table[1, 0], 0, 0] = bad
        got, lse = ops.PagedCache(k.cuda(), v.cuda()).attend(q.cuda(), table.cuda(), torch.tensor([n, 1], dtype=torch.int32, device="cuda"))
        close(got[0, :2], want[0, :2], bound[0, :2], "rows before")
        if victim is v:
            assert torch.isfinite(lse[:, 3]).all()
            out = got[1, 3].cpu().double()
            if q_t is cache_t:          # (else beyond the other type's range, or rounded to it)
                assert ((out - bad).abs() <= 2.0 ** -20 * abs(bad)).all()
        victim.copy_(kept)
    # no part of a key that a query has nothing in
    k.zero_()
    k[..., 0] = bad
    q.zero_()
    q[..., 1] = 1
    got, lse = ops.PagedCache(k.cuda(), v.cuda()).attend(q.cuda(), table.cuda(), torch.tensor([n, 1], dtype=torch.int32, device="cuda"))
    want, want_lse, weight, _ = ref.attend(q, k, v, table, [n, 1])
    close(got, want, UNIT[q_t] * want.abs() + (2.0 ** -11 + 2.0 ** -17) * weight + TINY[q_t], "queries of nothing")
    close(lse, want_lse, 2.0 ** -20 * want_lse.abs().nan_to_num(posinf=1.0) + 2.0 ** -20, "lse of nothing")


@pytest.mark.parametrize("bits", [0x7f800001, 0x7f800fff, 0x7fc00000, 0x7fffffff])
def test_attend_any_nan_of_fp32_pages_is_one(ops, bits):
    for victim in (0, 1):
        pool = [torch.zeros((1, 1, 32, 64)), torch.ones((1, 1, 32, 64))]
        pool[victim][0, 0, 4, 3] = torch.tensor(bits, dtype=torch.int32).view(F32)
        q = torch.ones((1, 1, 1, 64), device="cuda")
        got, _ = ops.PagedCache(pool[0].cuda(), pool[1].cuda()).attend(q, torch.zeros((1, 1), dtype=torch.int32, device="cuda"), torch.tensor([9], dtype=torch.int32, device="cuda"))
        assert got[0, 0, 0, 3].isnan()
        if victim:
            assert (got[0, 0, 0, 4:] == 1).all()


def test_calls_without_a_gradient_refuse_tensors_that_want_one(ops):
    kp = torch.zeros((4, 2, 32, 64), dtype=BF16, device="cuda")
    cache = ops.PagedCache(kp, kp.clone())
    table, one = torch.zeros((1, 4), dtype=torch.int32, device="cuda"), torch.ones(1, dtype=torch.int32, device="cuda")
    x = torch.zeros((1, 1, 2, 64), dtype=BF16, device="cuda")
    leaf = x.clone().requires_grad_()
    rope = ops.rope_table(8, 64)
    for call in (lambda: cache.append(leaf, x, table, one), lambda: cache.append(x, leaf, table, one), lambda: cache.append(x, x, table, one, q=leaf),
                 lambda: cache.append(x, x, table, one, q=2 * leaf, rope=rope), lambda: cache.append(x, x, table, one, q=x, out=2 * leaf),
                 lambda: cache.append(x, x, table, one, q=x, rope=rope.clone().requires_grad_()), lambda: cache.attend(leaf, table, one),
                 lambda: cache.attend(x, table, one, out=2 * leaf), lambda: cache.attend(cache.append(x, x, table, one, q=2 * leaf), table, one)):
        with pytest.raises(ValueError) as e:
            call()
        assert "no_grad" in str(e.value)
        with torch.no_grad():
            call()
    assert not cache.append(x, x, table, one, q=x).requires_grad


def test_numbers_beyond_their_type_are_refused(ops):
    from paper_2507_23777_b200.binding import XsmError
    kp = torch.zeros((4, 2, 32, 64), dtype=F16, device="cuda")
    cache = ops.PagedCache(kp, kp.clone())
    table, one = torch.zeros((1, 4), dtype=torch.int32, device="cuda"), torch.ones(1, dtype=torch.int32, device="cuda")
    q = torch.zeros((1, 1, 2, 64), dtype=F16, device="cuda")
    for call in (lambda: cache.attend(q, table, one, window=2 ** 31), lambda: cache.attend(q, table, one, window=1.5), lambda: cache.attend(q, table, one, scale=1e39)):
        with pytest.raises((ValueError, XsmError)):
            call()


def test_writes_in_place_are_seen_by_autograd(ops):
    """A tensor that another step keeps for its backward pass, written by a call: torch says so, as with its own operators."""
    kp = torch.zeros((4, 2, 32, 64), device="cuda")
    table, one = torch.zeros((1, 4), dtype=torch.int32, device="cuda"), torch.ones(1, dtype=torch.int32, device="cuda")
    w = torch.ones((), device="cuda", requires_grad=True)
    x = torch.ones((1, 1, 2, 64), device="cuda")
    z, t = torch.zeros((2, 10), device="cuda"), torch.zeros(2, dtype=torch.int64, device="cuda")

    def fresh():
        cache = ops.PagedCache(kp.clone(), kp.clone())
        return cache, cache.k, cache.v, x.clone(), torch.ones((1, 1, 2), device="cuda"), z.clone()
    for i, call in enumerate((lambda c, out, lse, d: c.append(x, x, table, one), lambda c, out, lse, d: c.append(x, x, table, one),
                              lambda c, out, lse, d: c.append(x, x, table, one, q=x, out=out), lambda c, out, lse, d: c.attend(x, table, one, out=out),
                              lambda c, out, lse, d: c.attend(x, table, one, lse=lse),
                              lambda c, out, lse, d: ops.token_logprobs_grad(d, t, ops.token_logprobs(d, t), out=d))):
        cache, k, v, out, lse, d = fresh()
        kept = (k, v, out, out, lse, d)[i]
        y = (w * kept).sum()
        with torch.no_grad():
            call(cache, out, lse, d)
        with pytest.raises(RuntimeError, match="modified by an inplace operation"):
            y.backward()


def recorded(calls):
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = calls()
    return graph, out


def test_a_wait_that_ran_out_in_a_graph_is_told(ops):
    """Status words of replays last until check, whichever of the recorded calls it was; good replays leave none."""
    from paper_2507_23777_b200.binding import XSM_ERR_TIMEOUT, XsmError
    g = gen(41)
    k, v, table = ref.pools(g, [700, 90], 2, 32, 64, F16)
    q = torch.randn((2, 3, 4, 64), generator=g).to(F16).cuda()
    cache, table, n = ops.PagedCache(k.cuda(), v.cuda()), table.cuda(), torch.tensor([700, 90], dtype=torch.int32, device="cuda")
    want, lse = cache.attend(q, table, n)
    good, (out, l2) = recorded(lambda: cache.attend(q, table, n))

    def bad_then_good():
        cache.lib.xsm_debug_kv_waits(cache._h, 20, 1)
        cache.attend(q, table, n)
        cache.lib.xsm_debug_kv_waits(cache._h, 0, 0)
        return cache.attend(q, table, n)
    bad, (out2, l3) = recorded(bad_then_good)
    good.replay()
    cache.check()
    assert torch.equal(out, want) and torch.equal(l2, lse)
    for _ in range(2):
        bad.replay()
        good.replay()
        with pytest.raises(XsmError) as e:
            cache.check()
        assert e.value.status == XSM_ERR_TIMEOUT
        assert torch.equal(out2, want) and torch.equal(l3, lse)
    good.replay()
    cache.check()


def test_recorded_calls_of_many_caches_share_a_workspace(ops):
    """One for a graph's calls on a stream, as large as the largest wants, in no graph's own memory; another graph has another; gone with its graph."""
    import gc
    g = gen(42)
    caches = []
    for d, hk in ((64, 2), (128, 1), (64, 2)):
        k, v, table = ref.pools(g, [1000, 90], hk, 32, d, F16)
        q = torch.randn((2, 3, 4, d), generator=g).to(F16).cuda()
        caches.append((ops.PagedCache(k.cuda(), v.cuda()), q, table.cuda()))
    n = torch.tensor([1000, 90], dtype=torch.int32, device="cuda")
    want = [c.attend(q, t, n)[0] for c, q, t in caches]
    gc.collect()
    before = set(ops._recorded)
    graphs = [recorded(lambda: [c.attend(q, t, n)[0] for c, q, t in caches]) for _ in range(2)]
    keys = [key for key in ops._recorded if key not in before]
    one, two = (ops._recorded[key] for key in keys)
    assert one.ws.data_ptr() != two.ws.data_ptr() and all(set(c._graphs) >= {one, two} for c, _, _ in caches)
    for _ in range(3):
        for graph, outs in graphs:
            [o.zero_() for o in outs]
            graph.replay()
            torch.cuda.synchronize()
            assert all(torch.equal(o, w) for o, w in zip(outs, want))
    # a graph does not need the caches to be kept, only the tensors of the calls and the pools
    kept = [(c.k, c.v, q, t) for c, q, t in caches]
    caches.clear(), gc.collect()
    others = [torch.full((one.size,), 85, dtype=torch.uint8, device="cuda") for _ in range(4)]
    for graph, outs in graphs:
        [o.zero_() for o in outs]
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(o, w) for o, w in zip(outs, want))
    assert all((o == 85).all() for o in others) and len(kept) == 3
    del one, two, graph, outs
    graphs.clear(), gc.collect(), torch.cuda.synchronize()
    import time
    for _ in range(100):          # (the driver says so from a thread of its own)
        ops._forget_graphs()
        if not any(key in ops._recorded for key in keys):
            break
        time.sleep(0.05)
    assert not any(key in ops._recorded for key in keys)


def test_graphs_and_calls_of_the_stream_that_they_were_recorded_on_side_by_side(ops):
    """Replays on other streams while the recording stream goes on with calls of its own, bit for bit."""
    g = gen(43)
    lens = [4000, 10, 2500, 900]
    k, v, table = ref.pools(g, lens, 2, 64, 64, F16)
    q = torch.randn((4, 5, 4, 64), generator=g).to(F16).cuda()
    cache, table, n = ops.PagedCache(k.cuda(), v.cuda()), table.cuda(), torch.tensor(lens, dtype=torch.int32, device="cuda")
    stream, other = torch.cuda.Stream(), torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(stream):
        want, lse = cache.attend(q, table, n)
    graphs = []
    for _ in range(2):
        graph = torch.cuda.CUDAGraph()
        torch.cuda.synchronize()
        with torch.cuda.graph(graph, stream=stream):
            graphs.append((graph, [cache.attend(q, table, n) for _ in range(5)]))
    torch.cuda.synchronize()
    calls = []
    for _ in range(10):
        graphs[0][0].replay()
        with torch.cuda.stream(other):
            graphs[1][0].replay()
        with torch.cuda.stream(stream):
            calls += [cache.attend(q, table, n) for _ in range(5)]
    torch.cuda.synchronize()
    for out, l2 in calls + graphs[0][1] + graphs[1][1]:
        assert torch.equal(out, want) and torch.equal(l2, lse)
    cache.check()


def test_append_many_tokens_of_many_heads(ops):
    """Prompts whose tokens have more elements than a block takes at once: 128 threads a token that go on to the next ones, in every type, width and
    pairing; ragged counts, parts of heads rotated, strides, pages that are not there."""
    def broken(table, n):
        table[0, 1], table[1, 0], table[1, 3] = -1, n, 2 ** 31 - 1
    for cache_t in (F32, BF16, F16):
        for in_t in (F32, BF16, F16):
            # (600 + 600 tokens; 24 heads of 64 are 96 items of sixteen elements, 768 pairs where the rotated part is no multiple of sixteen)
            for rot, interleaved in ((32, False), (32, True), (10, False), (64, True)):
                check_append(ops, cache_t, in_t, 64, 8, 8, 600, 64, [0, 37], rot=rot, interleaved=interleaved, counts=[600, 411], seed=rot + interleaved, break_table=broken)
    check_append(ops, F16, BF16, 128, 4, 0, 1100, 48, [5], rot=128, layout="nhd", seed=3)
    check_append(ops, BF16, BF16, 64, 16, 16, 513, 16, [0, 3], rot=None, seed=4, packed=False)


def test_append_few_tokens_of_more_items_than_threads(ops):
    """More than 512 items a token: 16 + 2 x 8 heads of 128 in pairs (2048), 64 + 2 x 8 heads of 128 in pieces (640)."""
    for cache_t in (F32, BF16, F16):
        for in_t in (F32, BF16, F16):
            for interleaved in (False, True):
                check_append(ops, cache_t, in_t, 128, 8, 16, 3, 32, [0, 31, 100], rot=10, interleaved=interleaved, counts=[3, 0, 2], seed=5)
                check_append(ops, cache_t, in_t, 128, 8, 64, 3, 32, [9, 90], rot=64, interleaved=interleaved, seed=6)


@pytest.mark.parametrize("m", [3, 600])
@pytest.mark.parametrize("rot,interleaved", [(64, False), (64, True), (10, False), (10, True)])
def test_append_queries_in_place(ops, m, rot, interleaved):
    """q_out = q gives what a tensor of its own gives, also where a thread takes item after item; tokens without a place or a count included."""
    g = gen(15)
    x = torch.randn((2, m, 24, 64), generator=g).to(F16).cuda()
    q, k, v = x.split([8, 8, 8], 2)
    pages = 2 * (-(-(m + 40) // 32)) + 1
    kp = torch.zeros((pages, 8, 32, 64), dtype=F16, device="cuda")
    table = torch.arange(pages - 1, dtype=torch.int32, device="cuda").view(2, -1)
    table[1, 0] = -1
    starts, counts = torch.tensor([40, -2], dtype=torch.int32, device="cuda"), torch.tensor([m, m - 1], dtype=torch.int32, device="cuda")
    rope = ops.rope_table(m + 39, rot)
    a, b = ops.PagedCache(kp, kp.clone()), ops.PagedCache(kp.clone(), kp.clone())
    want = a.append(k, v, table, starts, counts=counts, q=q, rope=rope, interleaved=interleaved)
    mine = x.clone()
    mq = mine[:, :, :8]
    assert b.append(k, v, table, starts, counts=counts, q=mq, rope=rope, interleaved=interleaved, out=mq) is mq
    assert torch.equal(mq, want) and torch.equal(mine[:, :, 8:], x[:, :, 8:]) and torch.equal(a.k, b.k) and torch.equal(a.v, b.v)
