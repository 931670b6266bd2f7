"""Gradients of the gated part and of head norms over tensors of more than 2^31 elements: rows at both ends and beyond the 2^31st, and sums over all of them in 64 bits."""
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


@pytest.mark.parametrize("dtype", [BF16, F16])
def test_gated_gradients_beyond_32_bits(ops, dtype):
    rows, ff, d, chunk = 2_100_003, 1032, 64, 60_000
    g = torch.Generator(device="cuda").manual_seed(1)
    x = torch.randn((rows, d), generator=g, device="cuda", dtype=dtype)
    wg, wu = ((1.5 * d ** -0.5 * torch.randn((ff, d), generator=g, device="cuda")).to(dtype) for _ in range(2))
    gy = torch.empty((rows, ff), device="cuda", dtype=dtype).normal_(generator=g)
    assert gy.numel() > 2 ** 31
    d_x, d_gate, d_up = ops.gated_feed_forward_grad(x, wg, wu, gy)
    sums = [[0.0, 0.0], [0.0, 0.0]]
    for a in range(0, rows, chunk):
        at = slice(a, min(a + chunk, rows))
        (want, bound), *more = ref.gated_grad(x[at], wg, wu, gy[at], "silu")
        near(d_x[at], want, bound, "d_x")
        for s, (v, b) in zip(sums, more):
            s[0], s[1] = s[0] + v, s[1] + b
    for v, (want, bound), what in zip((d_gate, d_up), sums, ("d_w_gate", "d_w_up")):
        near(v, want, bound * (rows / chunk + 1), what)        # (the accumulator holds all rows' sum while it takes the last of them)


def test_norm_gradients_beyond_32_bits(ops):
    m, heads, d, chunk = 2_100_003, 8, 128, 60_000
    g = torch.Generator(device="cuda").manual_seed(2)
    q = torch.empty((1, m, heads, d), device="cuda", dtype=BF16).normal_(generator=g)
    gq = torch.empty((1, m, heads, d), device="cuda", dtype=BF16).normal_(generator=g)
    assert q.numel() > 2 ** 31
    k, gk = q[:, :, :1], gq[:, :, 3:4]
    gains = [1 + 0.2 * torch.randn(d, generator=g, device="cuda") for _ in range(2)]
    positions = torch.randint(0, 1000, (1, m), generator=g, device="cuda").to(torch.int32)
    rope = ops.rope_table(999, d)          # (some are nowhere)
    got = ops.norm_rotate_grad(q, k, *gains, gq, gk, rope=rope, positions=positions)
    for i, (x, y) in enumerate(((q, gq), (k, gk))):
        want, bound, count = 0.0, 0.0, 0
        for a in range(0, m, chunk):
            at = slice(a, min(a + chunk, m))
            (dx, b), (dg, c) = ref.norm_grad(x[:, at], gains[i], y[:, at], rope, positions[:, at], 1e-6, False)
            near(got[i][:, at], dx, b, "d_" + "qk"[i])
            want, bound, count = want + dg, bound + c, count + 1
        near(got[2 + i], want, bound + want.abs() * 2.0 ** -24 * count, f"d_{'qk'[i]}_gain")
