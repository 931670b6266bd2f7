"""Log probabilities from hidden states, the gated feed-forward part and head norms: argument structures as the binding packs them, and refusals that need no device."""
import ctypes
import os
import subprocess

import pytest

from paper_2507_23777_b200 import binding, build

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
A = 4096          # an address that leads nowhere: nothing here touches a device


@pytest.fixture(scope="module")
def lib():
    build.build()
    return binding.load()


def test_structures_have_the_sizes_and_offsets_of_the_header(tmp_path):
    from paper_2507_23777_b200 import ops
    fields = {"xsm_linear_logprobs_args": ("hidden_stride", "workspace_bytes", "rows", "temperature"), "xsm_linear_logprobs_grad_args": ("hidden_stride", "workspace_bytes", "rows", "temperature"),
              "xsm_gated_ff_args": ("x_stride", "out_stride", "rows", "activation"), "xsm_gated_ff_grad_args": ("x_stride", "workspace_bytes", "rows", "activation"),
              "xsm_norm_rotate_args": ("q_stride", "k_out_stride", "batch", "eps"), "xsm_norm_rotate_grad_args": ("q_stride", "workspace_bytes", "batch", "eps"), "xsm_head_norm": ("gain_dtype", "eps")}
    src = tmp_path / "sizes.c"
    src.write_text('#include "xsm.h"\n#include <stdio.h>\n#include <stddef.h>\nint main(void) {\n' + "".join(
        f'printf("{t} %zu", sizeof({t}));' + "".join(f'printf(" %zu", offsetof({t}, {f}));' for f in fs) + 'puts("");' for t, fs in fields.items()) + "return 0; }\n")
    subprocess.check_call(["gcc", "-I", os.path.join(ROOT, "include"), str(src), "-o", str(tmp_path / "sizes")])
    got = {l.split()[0]: [int(x) for x in l.split()[1:]] for l in subprocess.check_output([str(tmp_path / "sizes")], text=True).splitlines()}

    def up(n):
        return (n + 7) // 8 * 8
    for name, s, pointers, strides in (("xsm_linear_logprobs_args", ops._LINEAR, 8, 4), ("xsm_linear_logprobs_grad_args", ops._LINEAR_GRAD, 11, 8), ("xsm_gated_ff_args", ops._GATED, 5, 4),
                                       ("xsm_gated_ff_grad_args", ops._GATED_GRAD, 10, 7)):
        assert got[name] == [up(s.size), 8 * pointers, 8 * (pointers + strides - 1), 8 * (pointers + strides), s.size - 4]
    assert got["xsm_norm_rotate_args"] == [up(ops._NORM.size), 64, 64 + 9 * 8, 64 + 12 * 8, ops._NORM.size - 4]
    assert got["xsm_norm_rotate_grad_args"] == [up(ops._NORM_GRAD.size), 112, 112 + 18 * 8, 112 + 19 * 8, ops._NORM_GRAD.size - 4]
    assert got["xsm_head_norm"] == [ops._HEAD_NORM.size, 16, 20]


def test_calls_without_arguments_are_refused(lib):
    for f in (lib.xsm_linear_logprobs, lib.xsm_linear_logprobs_grad, lib.xsm_gated_ff, lib.xsm_gated_ff_grad, lib.xsm_norm_rotate, lib.xsm_norm_rotate_grad):
        assert f(None, None) == binding.XSM_ERR_INVALID_ARG and b"null" in lib.xsm_last_error(None)
    assert lib.xsm_kv_append_norm(None, None, None, None) == binding.XSM_ERR_INVALID_ARG
    for f in (lib.xsm_linear_logprobs_workspace, lib.xsm_linear_logprobs_grad_workspace, lib.xsm_gated_ff_grad_workspace):
        assert f(0, 5, 8) == 0 and f(5, 0, 8) == 0 and f(-1, 5, 8) == 0
    assert lib.xsm_norm_rotate_grad_workspace(0) == 0 and lib.xsm_norm_rotate_grad_workspace(512) == 0


def linear(pointers=8 * [A], strides=(64, 64, 1), ws=1 << 30, rows=4, vocab=100, d=64, dtype=1, token_bytes=8, temperature=1.0):
    from paper_2507_23777_b200 import ops
    return ops._LINEAR.pack(*pointers, *strides, ws, rows, vocab, d, dtype, token_bytes, temperature)


@pytest.mark.parametrize("wrong,word", [(dict(dtype=0), b"dtype"), (dict(dtype=3), b"dtype"), (dict(rows=-1), b"rows"), (dict(vocab=0), b"vocab"), (dict(d=60, strides=(64, 64, 1)), b"d a positive"), (dict(d=0), b"d a positive"),
                                        (dict(token_bytes=2), b"token_bytes"), (dict(temperature=0.0), b"temperature"), (dict(temperature=float("nan")), b"temperature"),
                                        (dict(temperature=1e-45), b"temperature"), (dict(temperature=float("inf")), b"temperature"), (dict(strides=(60, 64, 1)), b"hidden"), (dict(strides=(64, 56, 1)), b"weight"),
                                        (dict(strides=(64, 65, 1)), b"weight"), (dict(pointers=[A + 2] + 7 * [A]), b"aligned"), (dict(pointers=[A, A, A + 4, A, A, A, A, A]), b"aligned"),
                                        (dict(pointers=5 * [A] + [A + 4, A, A]), b"aligned"), (dict(pointers=[0] + 7 * [A]), b"null"), (dict(pointers=6 * [A] + [0, A]), b"null")])
def test_wrong_arguments_of_linear_logprobs(lib, wrong, word):
    assert lib.xsm_linear_logprobs(linear(**wrong), None) == binding.XSM_ERR_INVALID_ARG
    assert word in lib.xsm_last_error(None)


def test_workspaces_that_are_too_small(lib):
    from paper_2507_23777_b200 import ops
    if lib.xsm_linear_logprobs_workspace(4, 100, 64) == 0:
        pytest.skip("sizes of workspaces go by the device")
    assert lib.xsm_linear_logprobs(linear(ws=0), None) == binding.XSM_ERR_CAPACITY
    args = ops._LINEAR_GRAD.pack(*11 * [A], 64, 64, 1, 1, 1, 64, 64, 0, 4, 100, 64, 1, 8, 1.0)
    assert lib.xsm_linear_logprobs_grad(args, None) == binding.XSM_ERR_CAPACITY
    args = ops._GATED_GRAD.pack(*10 * [A], 64, 64, 64, 100, 64, 64, 0, 4, 100, 64, 1, 0)
    assert lib.xsm_gated_ff_grad(args, None) == binding.XSM_ERR_CAPACITY


@pytest.mark.parametrize("wrong,word", [(dict(dtype=0), b"dtype"), (dict(rows=-1), b"rows"), (dict(ff=0), b"ff"), (dict(d=12), b"multiple"), (dict(activation=2), b"activation"), (dict(activation=-1), b"activation"),
                                        (dict(strides=(64, 64, 64, 99)), b"out"), (dict(strides=(68, 64, 64, 100)), b"aligned"), (dict(pointers=[A, A, A, A + 1, A]), b"out"), (dict(pointers=[A, A, 0, A, A]), b"null")])
def test_wrong_arguments_of_gated_ff(lib, wrong, word):
    from paper_2507_23777_b200 import ops
    c = dict(pointers=5 * [A], strides=(64, 64, 64, 100), rows=4, ff=100, d=64, dtype=1, activation=0)
    c.update(wrong)
    args = ops._GATED.pack(*c["pointers"], *c["strides"], c["rows"], c["ff"], c["d"], c["dtype"], c["activation"])
    assert lib.xsm_gated_ff(args, None) == binding.XSM_ERR_INVALID_ARG
    assert word in lib.xsm_last_error(None)


def test_sizes_beyond_what_tiles_are_counted_in(lib):
    from paper_2507_23777_b200 import ops
    big = (1 << 30) + 8
    for sizes in (dict(rows=big), dict(vocab=big), dict(d=big, strides=(big, big, 1))):
        assert lib.xsm_linear_logprobs(linear(**sizes), None) == binding.XSM_ERR_INVALID_ARG and b"2^30" in lib.xsm_last_error(None)
    for rows, ff, d in ((big, 8, 8), (8, big, 8), (8, 8, big)):
        args = ops._GATED.pack(*5 * [A], d, d, d, ff, rows, ff, d, 1, 0)
        assert lib.xsm_gated_ff(args, None) == binding.XSM_ERR_INVALID_ARG and b"2^30" in lib.xsm_last_error(None)
        assert lib.xsm_gated_ff_grad_workspace(rows, ff, d) == 0 == lib.xsm_linear_logprobs_grad_workspace(rows, ff, d)
    assert lib.xsm_linear_logprobs_workspace(big, 8, 8) == 0 == lib.xsm_linear_logprobs_workspace(8, big, 8)


def test_gradients_that_go_together(lib):
    from paper_2507_23777_b200 import ops
    args = ops._GATED_GRAD.pack(A, A, A, A, A, A, 0, A, A, A, 64, 64, 64, 100, 64, 64, 1 << 30, 4, 100, 64, 1, 0)
    assert lib.xsm_gated_ff_grad(args, None) == binding.XSM_ERR_INVALID_ARG and b"together" in lib.xsm_last_error(None)
    args = ops._GATED_GRAD.pack(A, A, A, A, 0, 0, 0, A, A, A, 64, 64, 64, 100, 64, 64, 1 << 30, 4, 100, 64, 1, 0)
    assert lib.xsm_gated_ff_grad(args, None) == 0          # nothing is wanted


@pytest.mark.parametrize("wrong,word", [(dict(dtype=3), b"types"), (dict(gain_dtype=-1), b"types"), (dict(d=48), b"d_head"), (dict(eps=-1.0), b"eps"), (dict(eps=float("nan")), b"eps"), (dict(rope=A, dims=0), b"rope_dims"),
                                        (dict(rope=A, dims=66), b"rope_dims"), (dict(rope=A, dims=3), b"rope_dims"), (dict(rope=A, dims=64, positions=0), b"rope"), (dict(rope=A + 4, dims=64, positions=9), b"aligned"),
                                        (dict(batch=-1), b"batch"), (dict(heads=5000), b"heads"), (dict(batch=1 << 20, m=1 << 20), b"2^31"), (dict(q=0), b"null"), (dict(q=A + 1), b"aligned")])
def test_wrong_arguments_of_norm_rotate(lib, wrong, word):
    from paper_2507_23777_b200 import ops
    c = dict(q=A, rope=0, batch=2, m=3, heads=4, d=64, dtype=1, gain_dtype=0, positions=9, dims=0, eps=1e-6)
    c.update(wrong)
    args = ops._NORM.pack(c["q"], A, A, A, A, A, 0, c["rope"], *4 * (768, 256, 64), c["batch"], c["m"], c["heads"], 2, c["d"], c["dtype"], c["gain_dtype"], c["positions"], c["dims"], 0, c["eps"])
    assert lib.xsm_norm_rotate(args, None) == binding.XSM_ERR_INVALID_ARG
    assert word in lib.xsm_last_error(None)
    args = ops._NORM_GRAD.pack(c["q"], A, A, A, 0, c["rope"], *8 * [A], *6 * (768, 256, 64), 1 << 30, c["batch"], c["m"], c["heads"], 2, c["d"], c["dtype"], c["gain_dtype"], c["positions"], c["dims"], 0, c["eps"])
    assert lib.xsm_norm_rotate_grad(args, None) == binding.XSM_ERR_INVALID_ARG
    assert word in lib.xsm_last_error(None)


def test_no_cpu_path():
    import torch
    if torch.cuda.is_available():
        pytest.skip("a GPU is present")
    from paper_2507_23777_b200 import ops
    x = torch.zeros(2, 8, dtype=torch.bfloat16)
    with pytest.raises((RuntimeError, ValueError)):
        ops.linear_logprobs(x, x, torch.zeros(2, dtype=torch.int64))
    with pytest.raises((RuntimeError, ValueError)):
        ops.gated_feed_forward(x, x, x)
    with pytest.raises((RuntimeError, ValueError)):
        ops.norm_rotate(torch.zeros(1, 1, 1, 32), None, torch.ones(32), None)


def test_divisions_by_a_product_and_a_shift():
    """The kernels divide numbers below 2^31 by umulhi(m, n) + n >> l: the same arithmetic, and the factor as the host makes it."""
    import random
    rng = random.Random(1)
    for _ in range(20000):
        d = rng.choice([rng.randrange(1, 50), rng.randrange(1, 1 << 30), 1 << rng.randrange(0, 31)])
        l = 0
        while l < 32 and (1 << l) < d:
            l += 1
        m = ((1 << 32) * ((1 << l) - d)) // d + 1
        assert m < 1 << 32
        for n in (rng.randrange(0, 1 << 31), d - 1, d, 0, (1 << 31) - 1, rng.randrange(0, 1 << 31) // d * d):
            assert (((m * n) >> 32) + n) % (1 << 32) >> l == n // d
