"""The operators' argument structures as the binding packs them, and refusals that need no device."""
import ctypes
import os
import subprocess

import pytest

from paper_2507_23777_b200 import binding, build

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def lib():
    build.build()
    return binding.load()


def test_structures_have_the_sizes_and_offsets_of_the_header(tmp_path):
    from paper_2507_23777_b200 import ops
    fields = {"xsm_kv_append_args": ("q_stride", "table_stride", "batch", "interleaved"),
              "xsm_kv_attend_args": ("q_stride", "workspace_bytes", "batch", "scale"),
              "xsm_logprob_args": ("row_stride", "rows", "temperature"),
              "xsm_logprob_grad_args": ("row_stride", "d_row_stride", "rows", "temperature"),
              "xsm_kv_config": ("row_stride", "n_pages", "dtype")}
    src = tmp_path / "sizes.c"
    src.write_text('#include "xsm.h"\n#include <stdio.h>\n#include <stddef.h>\nint main(void) {\n' + "".join(
        f'printf("{t} %zu", sizeof({t}));' + "".join(f'printf(" %zu", offsetof({t}, {f}));' for f in fs) + 'puts("");' for t, fs in fields.items()) +
        "return 0; }\n")
    subprocess.check_call(["gcc", "-I", os.path.join(ROOT, "include"), str(src), "-o", str(tmp_path / "sizes")])
    got = {l.split()[0]: [int(x) for x in l.split()[1:]] for l in subprocess.check_output([str(tmp_path / "sizes")], text=True).splitlines()}
    assert got["xsm_kv_append_args"] == [ops._APPEND.size, 64, 64 + 12 * 8, 64 + 13 * 8, ops._APPEND.size - 4]
    assert got["xsm_kv_attend_args"] == [ops._ATTEND.size, 56, 56 + 7 * 8, 56 + 8 * 8, ops._ATTEND.size - 4]
    assert got["xsm_logprob_args"] == [ops._LOGPROB.size, 56, 72, ops._LOGPROB.size - 4]
    assert got["xsm_logprob_grad_args"] == [ops._GRAD.size, 80, 120, 128, ops._GRAD.size - 4]
    assert got["xsm_kv_config"] == [ctypes.sizeof(binding.KvConfig), 16, 24, 40]


def test_calls_without_arguments_are_refused(lib):
    for status in (lib.xsm_kv_create(None, None, None, None), lib.xsm_kv_destroy(None), lib.xsm_kv_append(None, None, None), lib.xsm_kv_attend(None, None, None),
                   lib.xsm_token_logprobs(None, None), lib.xsm_token_logprobs_grad(None, None)):
        assert status == binding.XSM_ERR_INVALID_ARG
        assert b"null" in lib.xsm_last_error(None)
    assert lib.xsm_kv_attend_workspace(None, 1, 1, 1) == 0


def test_pools_that_do_not_fit_are_refused(lib):
    out = ctypes.c_void_p()
    good = dict(page_stride=2 * 32 * 64, head_stride=32 * 64, row_stride=64, n_pages=4, n_kv_heads=2, page_size=32, d_head=64, dtype=2)
    for wrong, word in ((dict(d_head=48), b"d_head"), (dict(page_size=24), b"page_size"), (dict(page_size=0), b"page_size"), (dict(dtype=3), b"dtype"), (dict(n_pages=0), b"n_pages"),
                        (dict(n_kv_heads=0), b"n_kv_heads"), (dict(row_stride=65), b"stride"), (dict(row_stride=32), b"stride"), (dict(page_stride=-4096), b"stride")):
        c = dict(good, **wrong)
        cfg = binding.KvConfig(*(c[n] for n, _ in binding.KvConfig._fields_))
        assert lib.xsm_kv_create(ctypes.byref(cfg), 4096, 4096, ctypes.byref(out)) == binding.XSM_ERR_INVALID_ARG, wrong
        assert word in lib.xsm_last_error(None) and not out.value
    cfg = binding.KvConfig(*(good[n] for n, _ in binding.KvConfig._fields_))
    assert lib.xsm_kv_create(ctypes.byref(cfg), 4098, 4096, ctypes.byref(out)) == binding.XSM_ERR_INVALID_ARG
    assert b"aligned" in lib.xsm_last_error(None)


def test_pointers_that_are_not_aligned_to_their_elements_are_refused(lib):
    """(Before anything touches a device: the addresses lead nowhere.)"""
    from paper_2507_23777_b200 import ops
    for logits, tokens in ((4097, 4096), (4096, 4100)):
        args = ops._LOGPROB.pack(logits, tokens, 4096, 4096, 4096, 0, 0, 64, 1, 2, 64, 1, 8, 0, 1.0)
        assert lib.xsm_token_logprobs(args, None) == binding.XSM_ERR_INVALID_ARG and b"aligned" in lib.xsm_last_error(None)
    args = ops._GRAD.pack(4096, 4096, 4096, 4096, 0, 4096, 0, 0, 0, 4097, 64, 1, 1, 0, 0, 64, 2, 64, 1, 8, 0, 1.0)
    assert lib.xsm_token_logprobs_grad(args, None) == binding.XSM_ERR_INVALID_ARG and b"aligned" in lib.xsm_last_error(None)


def test_no_cpu_path():
    import torch
    if torch.cuda.is_available():
        pytest.skip("a GPU is present")
    from paper_2507_23777_b200 import ops
    with pytest.raises((RuntimeError, ValueError)):
        ops.PagedCache(torch.zeros(1, 1, 16, 64), torch.zeros(1, 1, 16, 64))
    with pytest.raises((RuntimeError, ValueError)):
        ops.token_logprobs(torch.zeros(1, 8), torch.zeros(1, dtype=torch.int64))
