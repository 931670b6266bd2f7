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
import threading
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
_LINEAR = struct.Struct("8P4q5if")
_LINEAR_GRAD = struct.Struct("11P8q5if")
_GATED = struct.Struct("5P4q5i")
_GATED_GRAD = struct.Struct("10P7q5i")
_NORM = struct.Struct("8P12q10if")
_NORM_GRAD = struct.Struct("14P19q10if")
_HEAD_NORM = struct.Struct("2Pif")

TokenLogprobs = namedtuple("TokenLogprobs", "logprob entropy lse top_ids top_logprobs")
LinearLogprobs = namedtuple("LinearLogprobs", "logprob lse")

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


def _need_gain(g, d: int, device: int, dtype):
    _need(g.dim() == 1 and g.shape[0] == d and g.dtype is dtype and dtype in _DTYPES and g.stride(0) == 1 and g.get_device() == device,
          f"gains must be contiguous [{d}] on cuda:{device}, of fp32, bf16 or fp16, both of one type")


_empty = torch.empty_strided      # the quickest of torch's ways to new memory


def rope_table(n_positions: int, dims: int, theta: float = 10000.0, device="cuda"):
    """Cosine and sine of position * theta^(-2i/dims), computed in 64 bits: float32 [n_positions, dims / 2, 2]."""
    inv = float(theta) ** (-2.0 * torch.arange(dims // 2, dtype=torch.float64, device=device) / dims)
    angle = torch.arange(n_positions, dtype=torch.float64, device=device)[:, None] * inv
    return torch.stack([angle.cos(), angle.sin()], -1).float().contiguous()


class _Recorded:
    """The workspace of a graph's calls on one of its streams, outside of the graph's own memory: its status word outlasts a replay."""
    __slots__ = "ws", "size", "outgrown", "watch", "counter", "__weakref__"


_recorded = {}       # of graphs that exist: _Recorded by (device, number of the capture, stream)


def _forget_graphs():
    """Workspaces of graphs that are no more go back."""
    gone = binding.load().xsm_capture_gone
    for key in [key for key, r in list(_recorded.items()) if gone(r.watch)]:
        del _recorded[key]


def _zeros(n: int, device: int):
    """Zeroed memory that is kept from call to call; it may be written to in any mode, inference mode or not, whichever it is made in."""
    with torch.inference_mode(False):
        return torch.zeros(n, dtype=torch.uint8, device=f"cuda:{device}")


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
                t = _zeros(n, device)
            side.synchronize()
        finally:
            lib.xsm_capture_mode(before)
    return t


def _recorded_on(device: int, stream: int):
    """What belongs to the graph that is being recorded on the stream."""
    key = device, binding.load().xsm_capture_id(stream), stream
    r = _recorded.get(key)
    if r is None:
        _forget_graphs()
        r = _Recorded()
        r.ws, r.size, r.outgrown, r.watch, r.counter = None, 0, [], C.c_void_p(), None
        _check(binding.load().xsm_capture_watch(stream, C.byref(r.watch)))
        _recorded[key] = r
    return r


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

    def _gains(self, q, q_gain, k_gain, eps, rope):
        """The norm of an append as the library takes it."""
        _need(k_gain is not None and (q is None) == (q_gain is None), "gains go together: k_gain, and q_gain where there is q")
        dtype, d, device = k_gain.dtype, (self.d_head,), self.device
        ok = k_gain.shape == d and dtype in _DTYPES and k_gain.stride(0) == 1 and k_gain.get_device() == device
        if q_gain is not None:
            ok = ok and q_gain.shape == d and q_gain.dtype is dtype and q_gain.stride(0) == 1 and q_gain.get_device() == device
        if not ok:
            for g in (k_gain, q_gain):
                if g is not None:
                    _need_gain(g, self.d_head, device, dtype)
        _need(rope is None or rope.numel() > 0, "rope must not be empty")
        if _grad_enabled() and (k_gain.requires_grad or q_gain is not None and q_gain.requires_grad):
            raise ValueError("append has no gradient: call it under torch.no_grad()")
        if forward_ad._current_level >= 0:
            _no_tangents(k_gain, q_gain)
        try:
            return _HEAD_NORM.pack(0 if q_gain is None else q_gain.data_ptr(), k_gain.data_ptr(), _DTYPES[dtype], eps)
        except _BEYOND as e:
            raise ValueError(f"an argument of append is beyond its type: {e}") from None

    def append(self, k, v, block_table, starts, counts=None, q=None, rope=None, interleaved=False, out=None, q_gain=None, k_gain=None, eps=1e-6):
        """Writes k and v, [batch, m, n_kv_heads, d_head], to positions starts[b] + j (j < counts[b]) of every sequence; keys, and queries
        q [batch, m, n_heads, d_head], are rotated by `rope` (float32 [positions, dims / 2, 2], see rope_table).  Returns the rotated
        queries in `out` (a new tensor, or the one given; it may be q), or None without q.  With gains [d_head] (fp32, bf16 or fp16; q_gain where there is q)
        every head of keys and queries is normed before, as norm_rotate does it.  Like attend it has no gradient, and refuses tensors that
        want one unless torch.no_grad() says that it is not needed."""
        gains = None
        if k_gain is not None or q_gain is not None:
            gains = self._gains(q, q_gain, k_gain, eps, rope)
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
        status = self.lib.xsm_kv_append(self._h, args, _raw_stream(device)) if gains is None else self.lib.xsm_kv_append_norm(self._h, args, gains, _raw_stream(device))
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
            old, (ws, size) = ws, (_zeros(need, self.device), need)
            self._ws[stream] = ws, size
            if old is not None:
                self._outgrown.append(old)
        return ws, size

    def _workspace_of_graph(self, stream: int, need: int):
        r = _recorded_on(self.device, stream)
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


# ------------------------------------------------------------------------------------------ products with what follows them

_ACTIVATIONS = {"silu": 0, "gelu": 1}
_status_words = {}       # by device: a word that a wait that ran out leaves its status in


def _status(device: int, stream: int) -> int:
    """Address of the device's status word."""
    t = _status_words.get(device)
    if t is None:
        t = _zeros_while_recording(16, device) if stream and _capturing() else _zeros(16, device)
        t = _status_words.setdefault(device, t)          # (another thread may have been first)
    return t.data_ptr()


_counters = {}           # by (device, stream): words that calls count their CTAs in


def _counter(device: int, stream: int) -> int:
    """Address of words that are zero between the calls of a stream, or of a graph's on one of its streams."""
    if stream and _capturing():
        r = _recorded_on(device, stream)
        if r.counter is None:
            r.counter = _zeros_while_recording(4 * binding.XSM_COUNTERS, device)
        return r.counter.data_ptr()
    t = _counters.get((device, stream))
    if t is None:
        t = _counters.setdefault((device, stream), _zeros(4 * binding.XSM_COUNTERS, device))
    return t.data_ptr()


_KEPT = 1 << 20          # bytes of a workspace that is kept from call to call
_scratch_of = threading.local()
_sizes = {}              # by operator, device and sizes: bytes of its workspace, which go by the device's SMs


def _size_of(fn, device: int, *sizes) -> int:
    """What the library says of the current device."""
    n = _sizes.get((fn, device, sizes))
    if n is None:
        if len(_sizes) > 4096:
            _sizes.clear()
        n = _sizes[fn, device, sizes] = getattr(binding.load(), fn)(*sizes)
    return n


def _scratch(n: int, device: int, stream: int, where):
    """Memory for one call on the stream, of any content: a small one is the thread's from call to call, while nothing is recorded."""
    if n > _KEPT or stream and _capturing():
        return _empty((n,), (1,), dtype=torch.uint8, device=where)
    kept = _scratch_of.__dict__
    t = kept.get((device, stream))
    if t is None or t[1] < n:
        if len(kept) > 64:
            kept.clear()
        size = max(n, 1 << 16)
        t = kept[device, stream] = _empty((size,), (1,), dtype=torch.uint8, device=where), size
    return t[0]


def check(device=None):
    """Waits for the device (the current one) and raises an XsmError if a bounded wait of an earlier linear_logprobs, gated_feed_forward or gradient of
    theirs ran out there, replays of recorded ones among them (the results since the last check are void)."""
    i = device if device is None or isinstance(device, int) else torch.device(device).index
    if i is None:             # ("cuda" is the current one too)
        i = _current_device()
    torch.cuda.synchronize(i)
    t = _status_words.get(i)
    if t is not None:
        status = int(t[:4].view(torch.int32)[0])
        if status:
            t[:4].zero_()
            for c in [c for (d, _), c in list(_counters.items()) if d == i] + [r.counter for (d, _, _), r in list(_recorded.items()) if d == i and r.counter is not None]:
                c.zero_()          # (what gave up has not counted to the end)
            torch.cuda.synchronize(i)
            raise binding.XsmError(status, "a bounded device-side wait ran out of patience")


def _rows(t, what: str, device: int, dtype, width=None):
    """Row stride of a matrix of 16-bit elements that the products can take as it lies."""
    shape = t.shape
    if len(shape) != 2 or t.dtype is not dtype or width is not None and shape[1] != width:
        raise ValueError(f"{what} must be [rows, {'d' if width is None else width}] of {dtype}, not {list(shape)} of {t.dtype}")
    if t.get_device() != device:
        raise ValueError(f"{what} must be on cuda:{device}")
    n, w = shape
    ld, step = t.stride()
    if n < 2:
        ld = w
    if step != 1 and w > 1 or ld < w or ld & 7 or t.data_ptr() & 15:
        raise ValueError(f"rows of {what} must be of neighbouring elements, 16-byte aligned, and must not overlap")
    return ld


def _need_products(t, what: str):
    """Device and type of a call's first operand."""
    if t.dtype is not torch.bfloat16 and t.dtype is not torch.float16:
        raise ValueError(f"{what} must be of bf16 or fp16")
    device = t.get_device()
    if device < 0 or device != _current_device():
        _need_here(t)
    return device, t.dtype


def _no_gradient(what: str, *tensors):
    if _grad_enabled():
        for t in tensors:
            if t is not None and t.requires_grad:
                raise ValueError(f"{what} has no gradient of its own: call it under torch.no_grad()")
    if forward_ad._current_level >= 0:
        _no_tangents(*tensors)


def _refuse_linear(hidden, weight, tokens):
    """What is wrong with the arguments, told one by one."""
    device, dtype = _need_products(hidden, "hidden")
    _rows(hidden, "hidden", device, dtype)
    rows, d = hidden.shape
    _rows(weight, "weight", device, dtype, d)
    _need(d >= 8 and d % 8 == 0 and weight.shape[0] >= 1, "the width of hidden must be a positive multiple of 8, and weight must have rows")
    _need(tokens.shape == (rows,) and tokens.get_device() == device and tokens.dtype in _TOKENS, f"tokens must be int32 or int64 [{rows}] on cuda:{device}")
    raise ValueError("the arguments of linear_logprobs do not go together")


def _check_linear(hidden, weight, tokens):
    """(device, type, rows, d, row strides) of arguments that go together, all of it looked at at once."""
    shape, w_shape, dtype, device = hidden.shape, weight.shape, hidden.dtype, hidden.get_device()
    ok = len(shape) == 2 == len(w_shape) and (dtype is torch.bfloat16 or dtype is torch.float16)
    if ok:
        rows, d = shape
        (ld, a), (w_ld, b) = hidden.stride(), weight.stride()
        if rows < 2:
            ld = d
        if w_shape[0] < 2:
            w_ld = d
        ok = (w_shape[1] == d and d >= 8 and w_shape[0] >= 1 and (d | ld | w_ld) & 7 == 0 and a == b == 1 and ld >= d and w_ld >= d and weight.dtype is dtype and
              device == weight.get_device() == tokens.get_device() == _current_device() and tokens.shape == (rows,) and tokens.dtype in _TOKENS and
              (hidden.data_ptr() | weight.data_ptr()) & 15 == 0)
    if not ok:
        _refuse_linear(hidden, weight, tokens)
    return device, dtype, rows, d, ld, w_ld


def _linear_forward(hidden, weight, tokens, temperature, kept=None):
    """kept: a place for the log probabilities once more"""
    device, dtype, rows, d, ld, w_ld = _check_linear(hidden, weight, tokens)
    lib, where, vocab, stream = binding.load(), hidden.device, weight.shape[0], _raw_stream(device)
    logprob = _empty((rows,), (1,), dtype=torch.float32, device=where)
    lse = _empty((rows,), (1,), dtype=torch.float32, device=where)
    n = _size_of("xsm_linear_logprobs_workspace", device, rows, vocab, d)
    ws = _scratch(n, device, stream, where)
    try:
        args = _LINEAR.pack(hidden.data_ptr(), weight.data_ptr(), tokens.data_ptr(), logprob.data_ptr(), lse.data_ptr(), ws.data_ptr(), _status(device, stream),
                            _counter(device, stream) if rows <= 16 else 0, ld, w_ld, tokens.stride(0), n, rows, vocab, d, _DTYPES[dtype], _TOKENS[tokens.dtype], temperature)
    except _BEYOND as e:
        raise ValueError(f"an argument of linear_logprobs is beyond its type: {e}") from None
    status = lib.xsm_linear_logprobs_keep(args, 0 if kept is None else kept.data_ptr(), stream)
    if status:
        _check(status)
    return LinearLogprobs(logprob, lse)


def linear_logprobs_grad(hidden, weight, tokens, result, grad_logprob=None, grad_lse=None, temperature=1.0, need=(True, True)):
    """The gradients (d_hidden, d_weight), in their type, of sum(grad_logprob * logprob) + sum(grad_lse * lse) of what linear_logprobs returned as `result` for the
    same hidden, weight, tokens and temperature (the log probabilities may be None: a token's element of a probability next to 1 is then as good as lse tells).  grad_*: float32 [rows]; each
    may be missing.  need: which of the two are wanted; the other is None.  The logits are computed again, at most 256 MiB of their gradients (or 1024 tokens' of each row) are in memory at a
    time, rounded to the type (up to 128 rows or 64 tokens: held in two parts of it); in fp16 every row is scaled into its range there, rows 2^26 and more below the largest lose bits.  There
    are no second derivatives: tensors that want a gradient are refused unless torch.no_grad() says that it is not needed."""
    _no_gradient("linear_logprobs_grad", hidden, weight, *result, grad_logprob, grad_lse)
    device, dtype, rows, d, ld, w_ld = _check_linear(hidden, weight, tokens)
    logprob, lse = result
    for t in (lse,) if logprob is None else (lse, logprob):
        if t.shape != (rows,) or t.dtype is not torch.float32 or t.get_device() != device or rows > 1 and t.stride(0) != 1:
            raise ValueError("result must be what linear_logprobs returned for these hidden states")
    gl, gl_ld = _row_grad(grad_logprob, rows, device, "grad_logprob")
    gs, gs_ld = _row_grad(grad_lse, rows, device, "grad_lse")
    lib, where, vocab, stream = binding.load(), hidden.device, weight.shape[0], _raw_stream(device)
    d_hidden = _empty((rows, d), (d, 1), dtype=dtype, device=where) if need[0] else None
    d_weight = _empty((vocab, d), (d, 1), dtype=dtype, device=where) if need[1] else None
    n = _size_of("xsm_linear_logprobs_grad_workspace", device, rows, vocab, d)
    ws = _scratch(n, device, stream, where)
    try:
        args = _LINEAR_GRAD.pack(hidden.data_ptr(), weight.data_ptr(), tokens.data_ptr(), lse.data_ptr(), gl, gs, 0 if d_hidden is None else d_hidden.data_ptr(),
                                 0 if d_weight is None else d_weight.data_ptr(), ws.data_ptr(), _status(device, stream), _counter(device, stream), ld, w_ld, tokens.stride(0), gl_ld, gs_ld,
                                 d, d, n, rows, vocab, d, _DTYPES[dtype], _TOKENS[tokens.dtype], temperature)
    except _BEYOND as e:
        raise ValueError(f"an argument of linear_logprobs_grad is beyond its type: {e}") from None
    status = lib.xsm_linear_logprobs_grad_near(args, 0 if logprob is None else logprob.data_ptr(), stream)
    if status:
        _check(status)
    return d_hidden, d_weight


class _LinearLogprobs(torch.autograd.Function):
    @staticmethod
    def forward(ctx, hidden, weight, tokens, temperature):
        kept = torch.empty(hidden.shape[:1], dtype=torch.float32, device=hidden.device)        # (the caller may write to the log probabilities, to mask them for one)
        r = _linear_forward(hidden, weight, tokens, temperature, kept)
        ctx.save_for_backward(hidden, weight, tokens, kept, r.lse)
        ctx.temperature = temperature
        ctx.set_materialize_grads(False)
        return tuple(r)

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, g_logprob, g_lse):
        hidden, weight, tokens, *r = ctx.saved_tensors
        need = ctx.needs_input_grad[:2]
        if g_logprob is None and g_lse is None:
            return None, None, None, None
        return *linear_logprobs_grad(hidden, weight, tokens, r, g_logprob, g_lse, ctx.temperature, need), None, None


def linear_logprobs(hidden, weight, tokens, temperature: float = 1.0) -> LinearLogprobs:
    """Scores tokens [rows] (int32 or int64; one outside the vocabulary is none, and scores 0) under softmax(hidden weight^T / temperature) without keeping the
    logits: (logprob, lse) float32 [rows].  hidden [rows, d] and weight [vocab, d] of bf16 or fp16, d a multiple of 8, rows 16-byte aligned.  Differentiable by
    both, once and backwards."""
    if forward_ad._current_level >= 0:
        _no_tangents(hidden, weight)
    if _grad_enabled() and (hidden.requires_grad or weight.requires_grad):
        return LinearLogprobs(*_LinearLogprobs.apply(hidden, weight, tokens, temperature))
    return _linear_forward(hidden, weight, tokens, temperature)


def _refuse_gated(x, w_gate, w_up, activation):
    """What is wrong with the arguments, told one by one."""
    device, dtype = _need_products(x, "x")
    _need(x.dim() >= 1 and w_gate.dim() == 2 and w_gate.shape == w_up.shape, "x must be [..., d], w_gate and w_up [ff, d]")
    d = x.shape[-1]
    _need(d >= 8 and d % 8 == 0 and w_gate.shape[0] >= 1, "the width of x must be a positive multiple of 8, and w_gate and w_up must have rows")
    if activation not in _ACTIVATIONS:
        raise ValueError(f"activation must be one of {', '.join(_ACTIVATIONS)}, not {activation!r}")
    _rows(x.reshape(-1, d), "x", device, dtype)
    _rows(w_gate, "w_gate", device, dtype, d)
    _rows(w_up, "w_up", device, dtype, d)
    raise ValueError("the arguments of gated_feed_forward do not go together")


def _check_gated(x, w_gate, w_up, activation):
    """(device, type, x as a matrix, rows, ff, d, row strides) of arguments that go together, all of it looked at at once."""
    dtype, device, w_shape, kind = x.dtype, x.get_device(), w_gate.shape, _ACTIVATIONS.get(activation)
    ok = kind is not None and len(w_shape) == 2 and w_shape == w_up.shape and (dtype is torch.bfloat16 or dtype is torch.float16) and x.dim() >= 1
    if ok and x.shape[-1]:
        flat = x if x.dim() == 2 else x.reshape(-1, x.shape[-1])
        (rows, d), ff = flat.shape, w_shape[0]
        (ld, a), (g_ld, b), (u_ld, c) = flat.stride(), w_gate.stride(), w_up.stride()
        if rows < 2:
            ld = d
        if ff < 2:
            g_ld = u_ld = d
        ok = (w_shape[1] == d and d >= 8 and ff >= 1 and (d | ld | g_ld | u_ld) & 7 == 0 and a == b == c == 1 and ld >= d and g_ld >= d and u_ld >= d and
              w_gate.dtype is dtype is w_up.dtype and device == w_gate.get_device() == w_up.get_device() == _current_device() and
              (flat.data_ptr() | w_gate.data_ptr() | w_up.data_ptr()) & 15 == 0)
    else:
        ok = False
    if not ok:
        _refuse_gated(x, w_gate, w_up, activation)
    return device, dtype, flat, rows, ff, d, ld, g_ld, u_ld, kind


def _gated_forward(x, w_gate, w_up, activation):
    device, dtype, flat, rows, ff, d, ld, g_ld, u_ld, kind = _check_gated(x, w_gate, w_up, activation)
    stream = _raw_stream(device)
    out = _empty((rows, ff), (ff, 1), dtype=dtype, device=x.device) if flat is x else torch.empty((*x.shape[:-1], ff), dtype=dtype, device=x.device)
    try:
        args = _GATED.pack(flat.data_ptr(), w_gate.data_ptr(), w_up.data_ptr(), out.data_ptr(), _status(device, stream), ld, g_ld, u_ld, ff, rows, ff, d, _DTYPES[dtype], kind)
    except _BEYOND as e:
        raise ValueError(f"an argument of gated_feed_forward is beyond its type: {e}") from None
    status = binding.load().xsm_gated_ff(args, stream)
    if status:
        _check(status)
    return out


def gated_feed_forward_grad(x, w_gate, w_up, grad, activation: str = "silu", need=(True, True, True)):
    """The gradients (d_x, d_w_gate, d_w_up), in their type, of sum(grad * out) of what gated_feed_forward returned for the same arguments.  grad: like out,
    neighbouring elements in a row.  need: which are wanted (the last two go together); the others are None.  The gradients by gate and up are rounded to the type in the middle (up to
    128 rows or 32 columns: held in two parts of it); in fp16 every row is scaled into its range there, rows 2^26 and more below the largest lose bits.  There are no second derivatives: tensors that
    want a gradient are refused unless torch.no_grad() says that it is not needed."""
    _no_gradient("gated_feed_forward_grad", x, w_gate, w_up, grad)
    device, dtype, flat, rows, ff, d, ld, g_ld, u_ld, kind = _check_gated(x, w_gate, w_up, activation)
    g = grad
    if flat is not x:
        _need(grad.dim() >= 1 and grad.shape[:-1] == x.shape[:-1] and grad.shape[-1] == ff, f"grad must be {[*x.shape[:-1], ff]}")
        g = grad.reshape(-1, ff)
    if g.shape != (rows, ff) or g.dtype is not dtype or g.get_device() != device:
        raise ValueError(f"grad must be {[*x.shape[:-1], ff]} of {dtype} on cuda:{device}")
    gy_ld, step = g.stride()
    if step != 1 and ff > 1 and rows:
        raise ValueError("the elements of a row of grad must be neighbours")
    where, stream = x.device, _raw_stream(device)
    d_x = d_gate = d_up = None
    to_x = to_gate = to_up = 0
    need_x, need_gate, need_up = need
    if need_x:
        d_x = _empty((rows, d), (d, 1), dtype=dtype, device=where)
        to_x = d_x.data_ptr()
        if flat is not x:
            d_x = d_x.view(x.shape)
    if need_gate or need_up:
        d_gate, d_up = _empty((ff, d), (d, 1), dtype=dtype, device=where), _empty((ff, d), (d, 1), dtype=dtype, device=where)
        to_gate, to_up = d_gate.data_ptr(), d_up.data_ptr()
    n = _size_of("xsm_gated_ff_grad_workspace", device, rows, ff, d)
    ws = _scratch(n, device, stream, where)
    try:
        args = _GATED_GRAD.pack(flat.data_ptr(), w_gate.data_ptr(), w_up.data_ptr(), g.data_ptr(), to_x, to_gate, to_up, ws.data_ptr(), _status(device, stream), _counter(device, stream),
                                ld, g_ld, u_ld, gy_ld, d, d, n, rows, ff, d, _DTYPES[dtype], kind)
    except _BEYOND as e:
        raise ValueError(f"an argument of gated_feed_forward_grad is beyond its type: {e}") from None
    status = binding.load().xsm_gated_ff_grad(args, stream)
    if status:
        _check(status)
    return d_x, d_gate if need_gate else None, d_up if need_up else None


class _GatedFeedForward(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, w_gate, w_up, activation):
        ctx.save_for_backward(x, w_gate, w_up)
        ctx.activation = activation
        return _gated_forward(x, w_gate, w_up, activation)

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, g):
        x, w_gate, w_up = ctx.saved_tensors
        if g.stride(-1) != 1 or g.dim() > 2:
            g = g.contiguous()
        return *gated_feed_forward_grad(x, w_gate, w_up, g, ctx.activation, ctx.needs_input_grad[:3]), None


def gated_feed_forward(x, w_gate, w_up, activation: str = "silu"):
    """act(x w_gate^T) * (x w_up^T), [..., ff]: both projections, the activation ("silu" or "gelu") and the product in one kernel.  x [..., d], w_gate and w_up [ff, d]
    of bf16 or fp16, d a multiple of 8, rows 16-byte aligned; gate and up are held in fp32, the output is rounded once.  Differentiable by all three, once and
    backwards; nothing but the arguments is kept for that."""
    if forward_ad._current_level >= 0:
        _no_tangents(x, w_gate, w_up)
    if _grad_enabled() and (x.requires_grad or w_gate.requires_grad or w_up.requires_grad):
        return _GatedFeedForward.apply(x, w_gate, w_up, activation)
    return _gated_forward(x, w_gate, w_up, activation)


# --------------------------------------------------------------------------------------- norms of heads with the rotation

def _refuse_norm(q, k, q_gain, k_gain, rope, positions):
    """What is wrong with the arguments, told one by one."""
    _need((q is None) == (q_gain is None) and (k is None) == (k_gain is None) and (q is not None or k is not None),
          "q and q_gain go together, k and k_gain too, and one of the pairs must be there")
    x, gain = (q, q_gain) if q is not None else (k, k_gain)
    _need(x.dim() == 4 and x.dtype in _DTYPES, "q and k must be [batch, m, heads, d_head] of fp32, bf16 or fp16")
    _need_here(x)
    device = x.get_device()
    for t, g in ((q, q_gain), (k, k_gain)):
        if t is not None:
            _need(t.dim() == 4 and t.shape[:2] == x.shape[:2] and t.shape[3] == x.shape[3] and t.dtype is x.dtype and t.get_device() == device and t.stride(3) == 1,
                  "q and k must have the same batch, tokens, d_head, type and device, and neighbouring elements of a head")
            _need_gain(g, x.shape[3], device, gain.dtype)
    if rope is not None:
        _need(rope.dtype is torch.float32 and rope.dim() == 3 and rope.shape[2] == 2 and rope.numel() > 0 and rope.is_contiguous() and rope.get_device() == device,
              f"rope must be contiguous float32 [positions, dims / 2, 2] on cuda:{device}, and not empty")
    if positions is not None:
        _need(positions.shape == x.shape[:2] and positions.dtype is torch.int32 and positions.is_contiguous() and positions.get_device() == device,
              f"positions must be contiguous int32 {list(x.shape[:2])} on cuda:{device}")
    raise ValueError("the arguments of norm_rotate do not go together")


_NONE = 0, 0, 0, 0


def _norm_layout(q, k, q_gain, k_gain, rope, positions):
    """What goes into the arguments' structures, all of it looked at at once: (device, strides of q and of k, addresses, sizes and types)."""
    x, gain = (q, q_gain) if q is not None else (k, k_gain)
    if x is None or gain is None:
        _refuse_norm(q, k, q_gain, k_gain, rope, positions)
    shape, dtype, gain_dtype, device = x.shape, x.dtype, gain.dtype, x.get_device()
    ok = len(shape) == 4 and dtype in _DTYPES and gain_dtype in _DTYPES and device == _current_device()
    heads = kv_heads = n = half = to_q = to_k = to_qg = to_kg = to_rope = to_at = 0
    qs = ks = _NONE
    if ok:
        batch, m, _, d = shape
        if q is not None:
            qs, heads, to_q, to_qg = q.stride(), shape[2], q.data_ptr(), q_gain.data_ptr()
            ok = qs[3] == 1 and q_gain.shape == (d,) and q_gain.stride(0) == 1 and q_gain.get_device() == device
        if k is not None and k_gain is not None:
            ks, other, to_k, to_kg = k.stride(), k.shape, k.data_ptr(), k_gain.data_ptr()
            ok = (ok and len(other) == 4 and other[0] == batch and other[1] == m and other[3] == d and ks[3] == 1 and k.dtype is dtype and k.get_device() == device and
                  k_gain.shape == (d,) and k_gain.stride(0) == 1 and k_gain.dtype is gain_dtype and k_gain.get_device() == device)
            kv_heads = other[2] if ok else 0
        elif k is not None or k_gain is not None:
            ok = False
        if q is None and q_gain is not None:
            ok = False
        if rope is not None:
            r = rope.shape
            ok = ok and len(r) == 3 and r[2] == 2 and r[0] > 0 and r[1] > 0 and rope.dtype is torch.float32 and rope.is_contiguous() and rope.get_device() == device
            if ok:
                n, half, to_rope = r[0], r[1], rope.data_ptr()
        if positions is not None:
            ok = ok and positions.shape == (batch, m) and positions.dtype is torch.int32 and positions.is_contiguous() and positions.get_device() == device
            to_at = positions.data_ptr()
    if not ok:
        _refuse_norm(q, k, q_gain, k_gain, rope, positions)
    return device, qs, ks, (to_q, to_k, to_qg, to_kg, to_at, to_rope), (batch, m, heads, kv_heads, d, _DTYPES[dtype], _DTYPES[gain_dtype], n, 2 * half)


def _like(t):
    """A tensor like t whose heads' elements are neighbours, also where t's rows overlap."""
    r = torch.empty_like(t)
    return r if r.stride(3) == 1 else torch.empty(t.shape, dtype=t.dtype, device=t.device)


def _norm_forward(q, k, q_gain, k_gain, rope, positions, eps, interleaved):
    device, qs, ks, (to_q, to_k, to_qg, to_kg, to_at, to_rope), sizes = _norm_layout(q, k, q_gain, k_gain, rope, positions)
    q_out = k_out = None
    os = us = _NONE
    to_qo = to_ko = 0
    if q is not None:
        q_out = _like(q)
        os, to_qo = q_out.stride(), q_out.data_ptr()
    if k is not None:
        k_out = _like(k)
        us, to_ko = k_out.stride(), k_out.data_ptr()
    try:
        args = _NORM.pack(to_q, to_k, to_qo, to_ko, to_qg, to_kg, to_at, to_rope, qs[0], qs[1], qs[2], ks[0], ks[1], ks[2], os[0], os[1], os[2], us[0], us[1], us[2],
                          *sizes, interleaved, eps)
    except _BEYOND as e:
        raise ValueError(f"an argument of norm_rotate is beyond its type: {e}") from None
    status = binding.load().xsm_norm_rotate(args, _raw_stream(device))
    if status:
        _check(status)
    return q_out, k_out


def norm_rotate_grad(q, k, q_gain, k_gain, grad_q, grad_k, rope=None, positions=None, eps: float = 1e-6, interleaved: bool = False):
    """The gradients (d_q, d_k, d_q_gain, d_k_gain), in their types, of sum(grad_q * q') + sum(grad_k * k') of what norm_rotate returned for the same arguments; None
    beside what was not there.  There are no second derivatives: tensors that want a gradient are refused unless torch.no_grad() says that it is not
    needed."""
    _no_gradient("norm_rotate_grad", q, k, q_gain, k_gain, rope, grad_q, grad_k)
    device, qs, ks, (to_q, to_k, to_qg, to_kg, to_at, to_rope), sizes = _norm_layout(q, k, q_gain, k_gain, rope, positions)
    stream = _raw_stream(device)
    d_q = d_k = d_q_gain = d_k_gain = None
    gs = hs = os = us = _NONE
    to_g = to_h = to_dq = to_dk = to_dqg = to_dkg = 0
    ok = (q is None) == (grad_q is None) and (k is None) == (grad_k is None)
    if ok and q is not None:
        gs = grad_q.stride()
        ok = grad_q.shape == q.shape and grad_q.dtype is q.dtype and grad_q.get_device() == device and (gs[3] == 1 or grad_q.numel() == 0)
        d_q, d_q_gain = _like(q), torch.empty_like(q_gain) if sizes[2] else torch.zeros_like(q_gain)        # (heads: of none the library makes no sum)
        os, to_g, to_dq, to_dqg = d_q.stride(), grad_q.data_ptr(), d_q.data_ptr(), d_q_gain.data_ptr()
    if ok and k is not None:
        hs = grad_k.stride()
        ok = grad_k.shape == k.shape and grad_k.dtype is k.dtype and grad_k.get_device() == device and (hs[3] == 1 or grad_k.numel() == 0)
        d_k, d_k_gain = _like(k), torch.empty_like(k_gain) if sizes[3] else torch.zeros_like(k_gain)
        us, to_h, to_dk, to_dkg = d_k.stride(), grad_k.data_ptr(), d_k.data_ptr(), d_k_gain.data_ptr()
    if not ok:
        raise ValueError("grad_q and grad_k must be like q and k, with neighbouring elements of a head")
    size = _size_of("xsm_norm_rotate_grad_workspace", device, sizes[4])
    ws = _scratch(size, device, stream, d_q.device if q is not None else d_k.device)
    try:
        args = _NORM_GRAD.pack(to_q, to_k, to_qg, to_kg, to_at, to_rope, to_g, to_h, to_dq, to_dk, to_dqg, to_dkg, ws.data_ptr(), _counter(device, stream), qs[0], qs[1], qs[2], ks[0], ks[1], ks[2],
                               gs[0], gs[1], gs[2], hs[0], hs[1], hs[2], os[0], os[1], os[2], us[0], us[1], us[2], size, *sizes, interleaved, eps)
    except _BEYOND as e:
        raise ValueError(f"an argument of norm_rotate_grad is beyond its type: {e}") from None
    status = binding.load().xsm_norm_rotate_grad(args, stream)
    if status:
        _check(status)
    return d_q, d_k, d_q_gain, d_k_gain


class _NormRotate(torch.autograd.Function):
    @staticmethod
    def forward(ctx, q, k, q_gain, k_gain, rope, positions, eps, interleaved):
        ctx.save_for_backward(q, k, q_gain, k_gain, rope, positions)
        ctx.more = eps, interleaved
        ctx.set_materialize_grads(False)
        return _norm_forward(q, k, q_gain, k_gain, rope, positions, eps, interleaved)

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, g_q, g_k):
        q, k, q_gain, k_gain, rope, positions = ctx.saved_tensors
        if g_q is None and q is not None or g_k is None and k is not None:        # (what nothing came back for has no gradient)
            q, q_gain = (None, None) if g_q is None else (q, q_gain)
            k, k_gain = (None, None) if g_k is None else (k, k_gain)
        if q is None and k is None:
            return (None,) * 8
        g_q, g_k = (g if g is None or g.stride(3) == 1 else g.contiguous() for g in (g_q, g_k))
        d = norm_rotate_grad(q, k, q_gain, k_gain, g_q, g_k, rope, positions, *ctx.more)
        return *(x if need else None for x, need in zip(d, ctx.needs_input_grad)), None, None, None, None


def norm_rotate(q, k, q_gain, k_gain, rope=None, positions=None, eps: float = 1e-6, interleaved: bool = False):
    """Norms of queries and keys for each head with the rotation of the positions in the same pass: (q', k') with y = R (gain x / sqrt(mean(x^2) + eps)) over every head,
    q [batch, m, n_heads, d_head], k [batch, m, n_kv_heads, d_head] of fp32, bf16 or fp16 with neighbouring elements of a head, gains [d_head].  Token j of a sequence
    is at positions[sequence, j] (int32; without positions at j); rope (see rope_table) may be missing: no rotation.  Tokens at positions that the rope does not have
    come out as zero.  q and q_gain, or k and k_gain, may be None.  Differentiable by q, k and the gains, once and backwards."""
    if forward_ad._current_level >= 0:
        _no_tangents(q, k, q_gain, k_gain, rope)
    if _grad_enabled():
        if rope is not None and rope.requires_grad:
            raise ValueError("norm_rotate has no gradient by rope")
        for t in (q, k, q_gain, k_gain):
            if t is not None and t.requires_grad:
                return _NormRotate.apply(q, k, q_gain, k_gain, rope, positions, eps, interleaved)
    return _norm_forward(q, k, q_gain, k_gain, rope, positions, eps, interleaved)
