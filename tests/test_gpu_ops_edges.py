"""Calls of the operators on a caller's own activations and weights that are seldom made: from new threads, of nothing, on devices by their names."""
import threading

import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ops():
    assert torch.cuda.is_available(), "this test needs a B200"
    from paper_2507_23777_b200 import build, ops
    build.build()
    yield ops
    ops.check()


def on_a_new_thread(f):
    """What f returns on a thread that has made no call to the device yet; what it raises is raised here."""
    out = {}

    def run():
        try:
            out["r"] = f()
        except Exception as e:
            out["e"] = e
    t = threading.Thread(target=run)
    t.start()
    t.join()
    if "e" in out:
        raise out["e"]
    return out["r"]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("rows", [5, 300])
def test_first_calls_of_a_thread(ops, dtype, rows):
    """Nothing of the thread's has called the device before: the memory comes from torch's pool."""
    g = torch.Generator(device="cuda").manual_seed(0)
    x, gy = (torch.randn((rows, 64), generator=g, device="cuda").to(dtype) for _ in range(2))
    w = torch.randn((64, 64), generator=g, device="cuda").to(dtype)
    t = torch.randint(0, 64, (rows,), generator=g, device="cuda")
    gl = torch.randn(rows, generator=g, device="cuda")
    q, gain = torch.randn((1, rows, 2, 64), generator=g, device="cuda").to(dtype), torch.ones(64, device="cuda")
    pools = [torch.zeros((3, 2, 16, 64), device="cuda", dtype=dtype) for _ in range(2)]
    r = ops.linear_logprobs(x, w, t)
    calls = [lambda: ops.linear_logprobs(x, w, t), lambda: ops.linear_logprobs_grad(x, w, t, r, gl), lambda: [ops.gated_feed_forward(x, w, w)], lambda: ops.gated_feed_forward_grad(x, w, w, gy),
             lambda: ops.norm_rotate(q, q, gain, gain), lambda: ops.norm_rotate_grad(q, q, gain, gain, q, q), lambda: ops.PagedCache(*pools) and []]
    for f in calls:
        want = f()
        for _ in range(2):
            for a, b in zip(on_a_new_thread(f), want):
                assert torch.equal(a, b)


def test_a_backward_pass_that_is_the_first_call_of_autograds_thread():
    """In a process of its own: autograd's thread has not called the device before the gradient of the gated part."""
    import os
    import subprocess
    import sys
    code = """
import torch
from paper_2507_23777_b200 import ops
x, w = torch.randn(300, 64, device="cuda").bfloat16(), torch.randn(200, 64, device="cuda").bfloat16()
gy = torch.randn(300, 200, device="cuda").bfloat16()
want = [ops.gated_feed_forward_grad(x, w, w, gy) for _ in range(3)].pop()
x.requires_grad_()
out = ops.gated_feed_forward(x, w, w)
del want
got, = torch.autograd.grad(out, x, gy)
with torch.no_grad():
    assert torch.equal(got, ops.gated_feed_forward_grad(x, w, w, gy)[0])
"""
    subprocess.run([sys.executable, "-c", code], check=True, cwd=os.path.dirname(os.path.dirname(os.path.abspath(__file__))), timeout=300)


@pytest.mark.parametrize("heads,kv_heads", [(0, 2), (2, 0), (0, 0), (0, None), (None, 0)])
@pytest.mark.parametrize("batch,m", [(2, 3), (0, 3), (2, 0)])
def test_gains_of_no_heads_have_gradients_of_zero(ops, heads, kv_heads, batch, m):
    gains = [torch.ones(64, device="cuda"), torch.ones(64, device="cuda")]
    torch.full((8, 64), float("nan"), device="cuda")          # (what new memory may hold)
    x = [None if n is None else torch.ones((batch, m, n, 64), device="cuda") for n in (heads, kv_heads)]
    gains = [None if t is None else g for t, g in zip(x, gains)]
    for _ in range(3):
        d = ops.norm_rotate_grad(*x, *gains, *x)
        for n, t, dt, dg in zip((heads, kv_heads), x, d[:2], d[2:]):
            assert dt is None if t is None else dt.shape == t.shape
            if n == 0 or t is not None and batch * m == 0:
                assert (dg == 0).all()
            if dg is not None:
                dg.fill_(float("nan"))                         # (so does the memory of the next)
        del d, dt, dg


@pytest.mark.parametrize("shape", [(0, 3, 2, 64), (2, 0, 2, 64), (2, 3, 0, 64)])
def test_empty_batches_are_trained(ops, shape):
    """The gradient of a sum over nothing comes with strides of zero, which a copy of nothing keeps."""
    q, k = (torch.ones(shape, device="cuda", requires_grad=True) for _ in range(2))
    gains = [torch.ones(64, device="cuda", requires_grad=True) for _ in range(2)]
    a, b = ops.norm_rotate(q, k, *gains)
    d = torch.autograd.grad(a.sum() + b.sum(), [q, k, *gains])
    assert d[0].shape == d[1].shape == shape and (d[2] == 0).all() and (d[3] == 0).all()
    x = torch.ones((0, 4, 64), device="cuda", dtype=torch.bfloat16, requires_grad=True)
    w = torch.ones((72, 64), device="cuda", dtype=torch.bfloat16, requires_grad=True)
    d = torch.autograd.grad(ops.gated_feed_forward(x, w, w).sum(), [x, w])
    assert d[0].shape == x.shape and (d[1] == 0).all()
    d = torch.autograd.grad(ops.linear_logprobs(x.view(0, 64), w, torch.zeros(0, dtype=torch.int64, device="cuda")).logprob.sum(), [x, w])
    assert d[0].shape == x.shape and (d[1] == 0).all()


@pytest.mark.parametrize("device", [None, 0, "cuda", "cuda:0", torch.device("cuda"), torch.device("cuda", 0)])
def test_checks_of_a_device_by_any_of_its_names(ops, device):
    from paper_2507_23777_b200 import binding
    x = torch.ones((5, 64), device="cuda", dtype=torch.bfloat16)
    lib = binding.load()
    ops.check(device)
    try:
        lib.xsm_debug_product_waits(2000, 1)
        ops.gated_feed_forward(x, x, x)
        with pytest.raises(binding.XsmError, match="patience"):
            ops.check(device)
    finally:
        lib.xsm_debug_product_waits(0, 0)
    ops.check(device)


@pytest.mark.parametrize("first", ["score", "likelihood"])
def test_a_score_that_gave_up_says_nothing_of_the_next(ops, first):
    """Attention and products give up in the same score: the next one, of either kind, is told of neither."""
    import numpy as np

    from conftest import gpu_cfg
    from paper_2507_23777_b200 import binding, inputs, score
    cfg = gpu_cfg(dtype=1)
    s = score.Scorer(cfg, inputs.make_weights(cfg), 1, 40, library_products=True)
    cond, tokens = inputs.make_cond(cfg, 1), np.arange(40)[None]
    want = s.likelihood(cond, tokens).logprob
    lib = binding.load()
    try:
        lib.xsm_debug_product_waits(2000, 1)
        for c in s.cache:
            lib.xsm_debug_kv_waits(c._h, 2000, 1)
        with pytest.raises(binding.XsmError):
            getattr(s, first)(cond, tokens)
    finally:
        lib.xsm_debug_product_waits(0, 0)
        for c in s.cache:
            lib.xsm_debug_kv_waits(c._h, 0, 0)
    assert torch.equal(s.likelihood(cond, tokens).logprob, want)


def test_threads_that_share_a_stream(ops):
    """Counters are the stream's, scratch is a thread's: four threads' calls follow each other on one stream in any order."""
    stream = torch.cuda.Stream()
    work = []
    for i, dtype in enumerate((torch.bfloat16, torch.float16, torch.bfloat16, torch.float16)):
        g = torch.Generator(device="cuda").manual_seed(i)
        rows = (5, 300, 9000, 40)[i]
        h, w = (torch.randn((n, 64), generator=g, device="cuda").to(dtype) for n in (rows, 520))
        t = torch.randint(0, 520, (rows,), generator=g, device="cuda")
        gl, gy = torch.randn(rows, generator=g, device="cuda"), torch.randn((rows, 520), generator=g, device="cuda").to(dtype)
        q, gain = torch.randn((1, rows, 3, 64), generator=g, device="cuda").to(dtype), torch.ones(64, device="cuda")

        def calls(h=h, w=w, t=t, gl=gl, gy=gy, q=q, gain=gain):
            r = ops.linear_logprobs(h, w, t)
            return [*r, *ops.linear_logprobs_grad(h, w, t, r, gl), *ops.gated_feed_forward_grad(h, w, w, gy), *ops.norm_rotate_grad(q, q, gain, gain, q, q)]
        work.append((calls, calls()))
    torch.cuda.synchronize()
    go, out = threading.Barrier(len(work)), [None] * len(work)

    def run(i):
        try:
            with torch.cuda.stream(stream):
                go.wait()
                out[i] = [work[i][0]() for _ in range(20)]
        except Exception as e:
            out[i] = e
    threads = [threading.Thread(target=run, args=(i,)) for i in range(len(work))]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    torch.cuda.synchronize()
    for got, (_, want) in zip(out, work):
        assert not isinstance(got, Exception), got
        for x in got:
            assert all(torch.equal(a, b) for a, b in zip(x, want))


def test_gradients_of_a_decoding_heads_loss(ops):
    """A head's loss as its fitting takes it, hidden states and weights rounded to bf16 on the way: five tensors are rounded by 2^-8 of an element at most each, which bounds a gradient's norm, twice
    where it comes through both factors."""
    g = torch.Generator(device="cuda").manual_seed(3)
    x, w1, wo = torch.randn((500, 96), generator=g, device="cuda"), torch.randn((96, 96), generator=g, device="cuda") / 10, torch.randn((300, 96), generator=g, device="cuda") / 10
    t = torch.randint(0, 300, (500,), generator=g, device="cuda")
    leaves = [w1.clone().requires_grad_(), wo.clone().requires_grad_()]
    silu = torch.nn.functional.silu
    got = torch.autograd.grad(-ops.linear_logprobs((x + silu(x @ leaves[0].T)).bfloat16(), leaves[1].bfloat16(), t).logprob.mean(), leaves)
    wide = [v.double().requires_grad_() for v in (w1, wo)]
    want = torch.autograd.grad(torch.nn.functional.cross_entropy((x.double() + silu(x.double() @ wide[0].T)) @ wide[1].T, t), wide)
    for a, b in zip(got, want):
        assert float((a.double() - b).norm()) <= 10 * 2.0 ** -8 * float(b.norm())


@pytest.mark.parametrize("recorded", [False, True])
def test_waits_that_ran_out_in_inference_mode_are_told_outside(ops, monkeypatch, recorded):
    """What calls keep is made in inference mode here, and cleared outside of it."""
    from paper_2507_23777_b200 import binding
    monkeypatch.setattr(ops, "_status_words", {})
    monkeypatch.setattr(ops, "_counters", {})
    lib = binding.load()
    x = torch.ones((5, 64), device="cuda", dtype=torch.bfloat16)
    q = torch.ones((1, 2, 2, 64), device="cuda", dtype=torch.bfloat16)
    table, length = torch.zeros((1, 1), dtype=torch.int32, device="cuda"), torch.full((1,), 16, dtype=torch.int32, device="cuda")
    cache = ops.PagedCache(*(torch.ones((1, 2, 16, 64), device="cuda", dtype=torch.bfloat16) for _ in range(2)))

    def calls():
        ops.gated_feed_forward_grad(x, x, x, x[:, :5].contiguous())
        cache.attend(q, table, length)
    try:
        lib.xsm_debug_product_waits(2000, 1)
        lib.xsm_debug_kv_waits(cache._h, 2000, 1)
        with torch.inference_mode():
            if recorded:
                graph = torch.cuda.CUDAGraph()
                with torch.cuda.graph(graph):
                    calls()
                graph.replay()
            else:
                calls()
        for check in (ops.check, cache.check):
            with pytest.raises(binding.XsmError, match="patience"):
                check()
            check()
    finally:
        lib.xsm_debug_product_waits(0, 0)
        lib.xsm_debug_kv_waits(cache._h, 0, 0)
