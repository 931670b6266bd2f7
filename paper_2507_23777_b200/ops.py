"""Operators on a caller's own paged cache and on a caller's own logits: torch tensors in, torch tensors out.

`PagedCache` appends new tokens to pages of keys and values, rotated by their position on the way, and attends the newest tokens over
the pages.  `token_logprobs` scores given tokens (log probability, entropy, top alternatives) and is differentiable;
`token_logprobs_grad` is its gradient alone.  What each computes stands in include/xsm.h; every call is enqueued on torch's current
stream, waits for nothing and may be captured in a graph.  Arguments are checked here and in the library, before anything is launched: a
ValueError or an XsmError tells what is wrong.  There is no other path: without the library or a GPU the calls fail.
"""
from __future__ import annotations

import ctypes as C
import struct
import weakref
from collections import namedtuple

import torch
from torch.autograd import forward_ad

from . import binding

_DTYPES = {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}
_TOKENS = {torch.int64: 8, torch.int32: 4}
# the argument structures of include/xsm.h, packed in their order
_APPEND = struct.Struct("8P13q8i")
_ATTEND = struct.Struct("7P8q7if")
_LOGPROB = struct.Struct("7P2q5if")
_GRAD = struct.Struct("10P6q5if")

TokenLogprobs = namedtuple("TokenLogprobs", "logprob entropy lse top_ids top_logprobs")

_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (lambda i: torch.cuda.current_stream(i).cuda_stream)


# says to autograd that tensors have been written to: what keeps one of them for a backward pass notices
_written = torch._C._increment_version
_grad_enabled = torch.is_grad_enabled
_capturing = torch._C._cuda_isCurrentStreamCapturing
_current_device = getattr(torch._C, "_cuda_getDevice", None) or torch.cuda.current_device


_BEYOND = struct.error, OverflowError      # what packing says of a number that its field does not hold


def _check(status: int):
    if status:
        raise binding.XsmError(status, binding.load().xsm_last_error(None).decode())


def _need(ok, what: str):
    if not ok:
        raise ValueError(what)


def _no_tangents(*tensors):
    """Within a level of forward-mode differentiation: a tangent would get lost without a word."""
    for t in tensors:
        if t is not None and forward_ad.unpack_dual(t).tangent is not None:
            raise ValueError("the operators have no forward-mode derivatives")


def _need_here(t):
    """A tensor on the current device."""
    i = t.get_device()
    _need(i >= 0, "the tensors must be on a CUDA device; there is no CPU path")
    _need(i == _current_device(), f"the tensors are on cuda:{i}, which is not the current device")


def _need_ints(t, n: int, device: int, what: str):
    _need(t.dtype is torch.int32 and tuple(t.shape) == (n,) and (n < 2 or t.stride(0) == 1) and t.get_device() == device,
          f"{what} must be a contiguous int32 tensor of {n} elements on cuda:{device}")


_empty = torch.empty_strided      # the quickest of torch's ways to new memory


def rope_table(n_positions: int, dims: int, theta: float = 10000.0, device="cuda"):
    """Cosine and sine of position * theta^(-2i/dims), computed in 64 bits: float32 [n_positions, dims / 2, 2]."""
    inv = float(theta) ** (-2.0 * torch.arange(dims // 2, dtype=torch.float64, device=device) / dims)
    angle = torch.arange(n_positions, dtype=torch.float64, device=device)[:, None] * inv
    return torch.stack([angle.cos(), angle.sin()], -1).float().contiguous()


class _Recorded:
    """The workspace of a graph's calls on one of its streams, outside of the graph's own memory: its status word outlasts a replay."""
    __slots__ = "ws", "size", "outgrown", "watch", "__weakref__"


_recorded = {}       # of graphs that exist: _Recorded by (device, number of the capture, stream)


def _forget_graphs():
    """Workspaces of graphs that are no more go back."""
    gone = binding.load().xsm_capture_gone
    for key in [key for key, r in list(_recorded.items()) if gone(r.watch)]:
        del _recorded[key]


def _zeros_while_recording(n: int, device: int):
    """Zeroed memory that is no part of the graph that is being recorded, and ready when this returns."""
    lib = binding.load()
    with torch.cuda.device(device):
        before = lib.xsm_capture_mode(2)           # (relaxed: other streams may be waited for, memory may be made)
        try:
            side = torch.cuda.Stream()
            while lib.xsm_capture_id(side.cuda_stream):      # (torch hands its streams out in turn)
                side = torch.cuda.Stream()
            with torch.cuda.stream(side):
                t = torch.zeros(n, dtype=torch.uint8, device=f"cuda:{device}")
            side.synchronize()
        finally:
            lib.xsm_capture_mode(before)
    return t


class PagedCache:
    """Pools of keys and of values, [n_pages, n_kv_heads, page_size, d_head] (any strides with neighbouring elements in a row: a pool laid
    out [n_pages, page_size, n_kv_heads, d_head] is passed as its view `pool.transpose(1, 2)`).  fp32, bf16 or fp16; d_head 32, 64,
    96, 128 or 256; page_size a multiple of 16.  The tensors stay the caller's and are used in place.

    A block table is int32 [batch, max_pages]: position p of a sequence is row p % page_size of page table[sequence, p // page_size].
    Calls from several streams at a time are fine as far as the pools' contents allow it: every stream has a workspace of its own, and so has every
    graph (one for each of its streams, which all caches share and which lasts as long as the graph).  The pools, and the other tensors of recorded
    calls, are the caller's to keep."""

    def __init__(self, k, v):
        if not torch.cuda.is_available():
            raise RuntimeError("xsm needs a CUDA device; there is no CPU path")
        self._h = C.c_void_p()
        self.lib = binding.load()
        _need(k.dim() == 4 and k.dtype in _DTYPES, "the pools must be [n_pages, n_kv_heads, page_size, d_head] of fp32, bf16 or fp16")
        _need(v.shape == k.shape and v.dtype == k.dtype and v.stride() == k.stride() and v.device == k.device, "both pools must be alike")
        _need(k.stride(3) == 1, "the elements of a row must be neighbours")
        _need_here(k)
        self.device = k.get_device()
        self.k, self.v, self.dtype = k, v, k.dtype
        self.n_pages, self.n_kv_heads, self.page_size, self.d_head = k.shape
        cfg = binding.KvConfig(*(s if n > 1 else k.shape[3] for s, n in zip((k.stride(0), k.stride(1), k.stride(2)), k.shape)), *k.shape,
                               _DTYPES[k.dtype])
        self.scale = self.d_head ** -0.5
        self._ws, self._ws_bytes = {}, {}          # by stream: a workspace and its size; by shape of a call: what it needs
        self._outgrown = []                        # workspaces that larger ones took the place of: calls on their way may still write to them
        self._graphs = weakref.WeakSet()           # workspaces of graphs that calls of this cache were recorded in
        _check(self.lib.xsm_kv_create(C.byref(cfg), k.data_ptr(), v.data_ptr(), C.byref(self._h)))

    def __del__(self):
        h, self._h = getattr(self, "_h", None), None
        if h:
            self.lib.xsm_kv_destroy(h)

    # What is wrong with a call's arguments, told one by one.  (The calls look at all of it at once and come here when something is.)
    def _need_rows(self, x, what: str, heads=None):
        _need(x.dim() == 4 and x.shape[3] == self.d_head and (heads is None or x.shape[2] == heads),
              f"{what} must be [batch, m, {'n_heads' if heads is None else heads}, {self.d_head}], not {list(x.shape)}")
        _need_here(x)
        _need(x.get_device() == self.device, f"{what} must be on cuda:{self.device}")
        _need(x.stride(3) == 1, f"the elements of a head of {what} must be neighbours")

    def _need_table(self, table, batch: int):
        _need(table.dtype is torch.int32 and table.dim() == 2 and table.shape[0] == batch and table.get_device() == self.device and
              (table.shape[1] < 2 or table.stride(1) == 1), f"the block table must be int32 [{batch}, max_pages] on cuda:{self.device}")

    def _refuse_append(self, k, v, block_table, starts, counts, q, rope, out):
        self._need_rows(k, "k", self.n_kv_heads)
        self._need_rows(v, "v", self.n_kv_heads)
        _need(v.shape == k.shape and v.dtype is k.dtype and k.dtype in _DTYPES, "k and v must be alike, of fp32, bf16 or fp16")
        self._need_table(block_table, k.shape[0])
        _need_ints(starts, k.shape[0], self.device, "starts")
        if counts is not None:
            _need_ints(counts, k.shape[0], self.device, "counts")
        if q is not None:
            self._need_rows(q, "q")
            _need(q.shape[:2] == k.shape[:2] and q.dtype is k.dtype, "q must have the batch, the tokens and the type of k")
            self._need_rows(out, "out", q.shape[2])
            _need(out.shape == q.shape and out.dtype is q.dtype, "out must have the shape and the type of q")
        _need(rope is None or rope.dtype is torch.float32 and rope.dim() == 3 and rope.shape[2] == 2 and rope.is_contiguous() and
              rope.get_device() == self.device, f"rope must be contiguous float32 [positions, dims / 2, 2] on cuda:{self.device}")
        raise ValueError("the arguments of append do not go together")

    def _refuse_attend(self, q, block_table, lengths, counts, out, lse):
        self._need_rows(q, "q")
        _need(q.dtype in _DTYPES, "q must be of fp32, bf16 or fp16")
        self._need_table(block_table, q.shape[0])
        _need_ints(lengths, q.shape[0], self.device, "lengths")
        if counts is not None:
            _need_ints(counts, q.shape[0], self.device, "counts")
        self._need_rows(out, "out")
        _need(out.shape == q.shape and out.dtype is q.dtype, "out must have the shape and the type of q")
        n = list(q.shape[:3])
        _need(list(lse.shape) == n and lse.dtype is torch.float32 and lse.is_contiguous() and lse.get_device() == self.device,
              f"lse must be contiguous float32 {n} on cuda:{self.device}")
        raise ValueError("the arguments of attend do not go together")

    def append(self, k, v, block_table, starts, counts=None, q=None, rope=None, interleaved=False, out=None):
        """Writes k and v, [batch, m, n_kv_heads, d_head], to positions starts[b] + j (j < counts[b]) of every sequence; keys, and queries
        q [batch, m, n_heads, d_head], are rotated by `rope` (float32 [positions, dims / 2, 2], see rope_table).  Returns the rotated
        queries in `out` (a new tensor, or the one given; it may be q), or None without q.  Like attend it has no gradient, and refuses tensors that
        want one unless torch.no_grad() says that it is not needed."""
        if _grad_enabled() and (k.requires_grad or v.requires_grad or q is not None and q.requires_grad or rope is not None and rope.requires_grad or
                                        out is not None and out.requires_grad):
            raise ValueError("append has no gradient: call it under torch.no_grad()")
        if forward_ad._current_level >= 0:
            _no_tangents(k, v, q, rope)
        device, dtype, shape, ks, vs, table = self.device, k.dtype, k.shape, k.stride(), v.stride(), block_table.shape
        qs = os = (0, 0, 0, 1)
        heads = positions = half = 0
        ok = len(shape) == 4 and shape == v.shape and len(table) == 2 and dtype in _DTYPES
        if ok:
            batch, m, kv_heads, d = shape
            ok = (kv_heads == self.n_kv_heads and d == self.d_head and ks[3] == vs[3] == 1 and v.dtype is dtype and table[0] == batch and
                  starts.shape == (batch,) and block_table.dtype is starts.dtype is torch.int32 and k.get_device() == device == v.get_device() and
                  block_table.get_device() == device == starts.get_device() == _current_device())
        if ok and q is not None:
            qs, q_shape = q.stride(), q.shape
            if out is None:
                out = torch.empty(q_shape, dtype=q.dtype, device=q.device)
            os = out.stride()
            ok = (len(q_shape) == 4 and q_shape == out.shape and qs[3] == os[3] == 1 and q_shape[0] == batch and q_shape[1] == m and q_shape[3] == d and
                  q.dtype is dtype is out.dtype and q.get_device() == device == out.get_device())
            if ok:
                heads = q_shape[2]
        else:
            out = None if q is None else out
        if ok and rope is not None:
            r = rope.shape
            ok = len(r) == 3 and r[2] == 2 and rope.dtype is torch.float32 and rope.is_contiguous() and rope.get_device() == device
            if ok:
                positions, half, _ = r
        if ok:
            ts = block_table.stride()
            ok = (table[1] < 2 or ts[1] == 1) and (batch < 2 or starts.stride(0) == 1)
        if ok and counts is not None:
            ok = counts.shape == (batch,) and counts.dtype is torch.int32 and counts.get_device() == device and (batch < 2 or counts.stride(0) == 1)
        if not ok:
            self._refuse_append(k, v, block_table, starts, counts, q, rope, out if out is not None else q)
        try:
            args = _APPEND.pack(
                0 if q is None else q.data_ptr(), k.data_ptr(), v.data_ptr(), 0 if out is None else out.data_ptr(), block_table.data_ptr(),
                starts.data_ptr(), 0 if counts is None else counts.data_ptr(), 0 if rope is None else rope.data_ptr(),
                qs[0], qs[1], qs[2], ks[0], ks[1], ks[2], vs[0], vs[1], vs[2], os[0], os[1], os[2], ts[0],
                batch, m, heads, _DTYPES[dtype], table[1], positions, 2 * half, interleaved)
        except _BEYOND as e:
            raise ValueError(f"an argument of append is beyond its type: {e}") from None
        _written((self.k, self.v) if out is None else (self.k, self.v, out))
        status = self.lib.xsm_kv_append(self._h, args, _raw_stream(device))
        if status:
            _check(status)
        return out

    def _workspace(self, stream: int, batch: int, m: int, heads: int):
        """Zeroed memory for the calls of a stream, kept from call to call, or for those of a graph."""
        need = self._ws_bytes.get((batch, m, heads))
        if need is None:
            need = self._ws_bytes[batch, m, heads] = max(16, self.lib.xsm_kv_attend_workspace(self._h, batch, m, heads))
        if stream and _capturing():               # (the default stream, 0, cannot be recorded)
            return self._workspace_of_graph(stream, need)
        ws, size = self._ws.get(stream, (None, 0))
        if size < need:
            old, (ws, size) = ws, (torch.zeros(need, dtype=torch.uint8, device=self.k.device), need)
            self._ws[stream] = ws, size
            if old is not None:
                self._outgrown.append(old)
        return ws, size

    def _workspace_of_graph(self, stream: int, need: int):
        key = self.device, self.lib.xsm_capture_id(stream), stream
        r = _recorded.get(key)
        if r is None:
            _forget_graphs()
            r = _Recorded()
            r.ws, r.size, r.outgrown, r.watch = None, 0, [], C.c_void_p()
            _check(self.lib.xsm_capture_watch(stream, C.byref(r.watch)))
            _recorded[key] = r
        if r.size < need:
            ws = _zeros_while_recording(need, self.device)
            if r.ws is not None:
                r.outgrown.append(r.ws)            # calls that are recorded already write to it
            r.ws, r.size = ws, need
        self._graphs.add(r)
        return r.ws, r.size

    def check(self):
        """Waits for the device and raises an XsmError if a bounded wait of an earlier attend ran out (its results are void): one of this cache, or
        one in a graph that calls of this cache were recorded in."""
        torch.cuda.synchronize(self.device)
        for ws in [ws for ws, _ in self._ws.values()] + self._outgrown + [ws for r in list(self._graphs) if r.ws is not None for ws in (r.ws, *r.outgrown)]:
            status = int(ws[:4].view(torch.int32)[0])
            if status:
                ws[:4].zero_()
                raise binding.XsmError(status, "a bounded device-side wait ran out of patience")

    def attend(self, q, block_table, lengths, counts=None, causal=True, window=0, scale=None, out=None, lse=None):
        """Attention of the newest tokens: q [batch, m, n_heads, d_head] over the first lengths[b] positions of every sequence, the new ones
        included.  Query j of n = counts[b] (m without counts) sees positions up to lengths[b] - n + j (all with causal=False), and
        of these the last `window` (0: all).  Returns (out, lse): out like q, lse float32 [batch, m, n_heads], the logarithm of the sum
        of exp(scale q.k), -inf where nothing is seen."""
        device, shape, qs, dtype, table = self.device, q.shape, q.stride(), q.dtype, block_table.shape
        if _grad_enabled() and (q.requires_grad or out is not None and out.requires_grad or lse is not None and lse.requires_grad):
            raise ValueError("attend has no gradient: call it under torch.no_grad()")
        if forward_ad._current_level >= 0:
            _no_tangents(q, self.k, self.v)
        if out is None:
            out = torch.empty(shape, dtype=dtype, device=q.device)
        rows = shape[:3]
        if lse is None:
            lse = torch.empty(rows, dtype=torch.float32, device=q.device)
        os = out.stride()
        ok = len(shape) == 4 and len(table) == 2 and shape == out.shape and lse.shape == rows and dtype in _DTYPES
        if ok:
            batch, m, heads, d = shape
            ts = block_table.stride()
            ok = (d == self.d_head and qs[3] == os[3] == 1 and table[0] == batch and (table[1] < 2 or ts[1] == 1) and lengths.shape == (batch,) and
                  (batch < 2 or lengths.stride(0) == 1) and out.dtype is dtype and lse.dtype is torch.float32 and lse.is_contiguous() and
                  block_table.dtype is lengths.dtype is torch.int32 and q.get_device() == device == out.get_device() == lse.get_device() and
                  block_table.get_device() == device == lengths.get_device() == _current_device())
        if ok and counts is not None:
            ok = counts.shape == (batch,) and counts.dtype is torch.int32 and counts.get_device() == device and (batch < 2 or counts.stride(0) == 1)
        if not ok:
            self._refuse_attend(q, block_table, lengths, counts, out, lse)
        stream = _raw_stream(device)
        ws, ws_bytes = self._workspace(stream, batch, m, heads)
        try:
            args = _ATTEND.pack(
                q.data_ptr(), out.data_ptr(), lse.data_ptr(), block_table.data_ptr(), lengths.data_ptr(), 0 if counts is None else counts.data_ptr(),
                ws.data_ptr(), qs[0], qs[1], qs[2], os[0], os[1], os[2], ts[0], ws_bytes, batch, m, heads, _DTYPES[dtype], table[1], causal, window,
                self.scale if scale is None else scale)
        except _BEYOND as e:
            raise ValueError(f"an argument of attend is beyond its type: {e}") from None
        _written((out, lse))
        status = self.lib.xsm_kv_attend(self._h, args, stream)
        if status:
            _check(status)
        return out, lse


def _check_logits(logits, tokens):
    """(device, rows, vocab, row stride, token stride) of arguments that go together."""
    device, shape = logits.get_device(), logits.shape
    if len(shape) != 2 or logits.dtype not in _DTYPES:
        raise ValueError("logits must be [rows, vocab] of fp32, bf16 or fp16")
    rows, vocab = shape
    ld, step = logits.stride()
    if step != 1 and vocab > 1:
        raise ValueError("the logits of a row must be neighbours")
    if device < 0 or device != _current_device():
        _need_here(logits)
    if tokens.shape != (rows,) or tokens.get_device() != device or tokens.dtype not in _TOKENS:
        raise ValueError(f"tokens must be int32 or int64 [{rows}] on cuda:{device}")
    return device, rows, vocab, ld, tokens.stride(0)


def _forward(logits, tokens, top, temperature):
    device, rows, vocab, ld, token_ld = _check_logits(logits, tokens)
    where, f32, row = logits.device, torch.float32, (rows,)
    logprob = _empty(row, (1,), dtype=f32, device=where)
    entropy = _empty(row, (1,), dtype=f32, device=where)
    lse = _empty(row, (1,), dtype=f32, device=where)
    ids = alt = None
    to_ids = to_alt = 0
    if top > 0:
        if top > min(32, vocab) or top != int(top):
            raise ValueError(f"top must be a whole number in [0, 32] and at most vocab, not {top}")
        ids = _empty((rows, top), (top, 1), dtype=torch.int32, device=where)
        alt = _empty((rows, top), (top, 1), dtype=f32, device=where)
        to_ids, to_alt = ids.data_ptr(), alt.data_ptr()
    try:
        args = _LOGPROB.pack(
            logits.data_ptr(), tokens.data_ptr(), logprob.data_ptr(), entropy.data_ptr(), lse.data_ptr(), to_ids, to_alt,
            ld, token_ld, rows, vocab, _DTYPES[logits.dtype], _TOKENS[tokens.dtype], top, temperature)
    except _BEYOND as e:
        raise ValueError(f"an argument of token_logprobs is beyond its type: {e}") from None
    status = binding.load().xsm_token_logprobs(args, _raw_stream(device))
    if status:
        _check(status)
    return TokenLogprobs(logprob, entropy, lse, ids, alt)


def _row_grad(g, rows, device, what):
    if g is None:
        return 0, 0
    if g.shape != (rows,) or g.dtype is not torch.float32 or g.get_device() != device:
        raise ValueError(f"{what} must be float32 [{rows}] on cuda:{device}")
    return g.data_ptr(), g.stride(0)


def token_logprobs_grad(logits, tokens, result, grad_logprob=None, grad_entropy=None, grad_lse=None, grad_top=None, temperature=1.0, out=None):
    """The gradient by the logits, in their type, of sum(grad_logprob * logprob) + sum(grad_entropy * entropy) + ... of what token_logprobs
    returned as `result` for the same logits, tokens and temperature.  grad_*: float32 [rows], grad_top [rows, top]; each may be
    missing.  out: a tensor like logits for the gradient, which may be the logits themselves.  There are no second derivatives: tensors that want a
    gradient are refused unless torch.no_grad() says that it is not needed."""
    device, rows, vocab, ld, token_ld = _check_logits(logits, tokens)
    if _grad_enabled():
        for t in (logits, result[2], grad_logprob, grad_entropy, grad_lse, grad_top, out):
            if t is not None and t.requires_grad:
                raise ValueError("token_logprobs_grad has no gradient of its own: call it under torch.no_grad()")
    if forward_ad._current_level >= 0:
        _no_tangents(logits, grad_logprob, grad_entropy, grad_lse, grad_top)
    if out is None:
        out = _empty((rows, vocab), (vocab, 1), dtype=logits.dtype, device=logits.device)
    elif out.shape != logits.shape or out.dtype is not logits.dtype or out.get_device() != device or out.stride(1) != 1 and vocab > 1 or \
            out.stride(0) < vocab and rows > 1:
        raise ValueError("out must be like logits, with rows of their own")
    else:
        _written([out])
    logprob, entropy, lse, ids, _ = result
    if not (lse.shape == entropy.shape == logprob.shape == (rows,) and lse.dtype is entropy.dtype is logprob.dtype is torch.float32 and
            lse.get_device() == device == entropy.get_device() and logprob.get_device() == device and
            lse.is_contiguous() and entropy.is_contiguous() and logprob.is_contiguous()):
        raise ValueError("result must be what token_logprobs returned for these logits")
    gl, gl_ld = _row_grad(grad_logprob, rows, device, "grad_logprob")
    ge, ge_ld = _row_grad(grad_entropy, rows, device, "grad_entropy")
    gs, gs_ld = _row_grad(grad_lse, rows, device, "grad_lse")
    top = alternatives = gt = 0
    if grad_top is not None:
        if ids is None or grad_top.shape != ids.shape or grad_top.dtype is not torch.float32 or not grad_top.is_contiguous() or \
                grad_top.get_device() != device or ids.shape[0] != rows or ids.dtype is not torch.int32 or not ids.is_contiguous() or \
                ids.get_device() != device:
            raise ValueError("grad_top must be contiguous float32 [rows, top] beside the result's top_ids")
        top, alternatives, gt = ids.shape[1], ids.data_ptr(), grad_top.data_ptr()
    try:
        args = _GRAD.pack(
            logits.data_ptr(), tokens.data_ptr(), lse.data_ptr(), entropy.data_ptr(), alternatives, gl, ge, gs, gt, out.data_ptr(),
            ld, token_ld, gl_ld, ge_ld, gs_ld, out.stride(0), rows, vocab, _DTYPES[logits.dtype], _TOKENS[tokens.dtype], top, temperature)
    except _BEYOND as e:
        raise ValueError(f"an argument of token_logprobs_grad is beyond its type: {e}") from None
    status = binding.load().xsm_token_logprobs_grad_near(args, logprob.data_ptr(), _raw_stream(device))
    if status:
        _check(status)
    return out


class _TokenLogprobs(torch.autograd.Function):
    @staticmethod
    def forward(ctx, logits, tokens, top, temperature):
        r = _forward(logits, tokens, top, temperature)
        ctx.save_for_backward(logits, tokens, *r)
        ctx.temperature = temperature
        ctx.set_materialize_grads(False)
        if r.top_ids is not None:
            ctx.mark_non_differentiable(r.top_ids)
        return tuple(r)

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, g_logprob, g_entropy, g_lse, _, g_top):
        logits, tokens, *r = ctx.saved_tensors
        if g_logprob is None and g_entropy is None and g_lse is None and g_top is None:
            return None, None, None, None
        d = token_logprobs_grad(logits, tokens, TokenLogprobs(*r), g_logprob, g_entropy, g_lse,
                                None if g_top is None else g_top.contiguous(), ctx.temperature)
        return d, None, None, None


def token_logprobs(logits, tokens, top: int = 0, temperature: float = 1.0) -> TokenLogprobs:
    """Scores tokens [rows] (int32 or int64; one outside the vocabulary is none, and scores 0) under softmax(logits / temperature), logits
    [rows, vocab]: (logprob, entropy, lse) float32 [rows], and with `top` > 0 the ids (int32 [rows, top]) and log probabilities of the
    largest logits, equal ones by the lower id first.  Differentiable by the logits, once and backwards."""
    if forward_ad._current_level >= 0:
        _no_tangents(logits)
    if logits.requires_grad and _grad_enabled():
        return TokenLogprobs(*_TokenLogprobs.apply(logits, tokens, top, temperature))
    return _forward(logits, tokens, top, temperature)
