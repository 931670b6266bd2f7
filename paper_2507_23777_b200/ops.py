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
from collections import namedtuple

import torch

from . import binding

_DTYPES = {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}
# the argument structures of include/xsm.h, packed in their order
_APPEND = struct.Struct("8P13q8i")
_ATTEND = struct.Struct("7P8q7if")
_LOGPROB = struct.Struct("7P2q5if")
_GRAD = struct.Struct("10P6q5if")

TokenLogprobs = namedtuple("TokenLogprobs", "logprob entropy lse top_ids top_logprobs")

_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (lambda i: torch.cuda.current_stream(i).cuda_stream)


def _check(status: int):
    if status:
        raise binding.XsmError(status, binding.load().xsm_last_error(None).decode())


def _need(ok, what: str):
    if not ok:
        raise ValueError(what)


def _ptr(t):
    return 0 if t is None else t.data_ptr()


def _here(t) -> int:
    """The index of a tensor's device, which has to be the current one."""
    i = t.get_device()
    if i < 0:
        raise ValueError("the tensors must be on a CUDA device; there is no CPU path")
    if i != torch.cuda.current_device():
        raise ValueError(f"the tensors are on cuda:{i}, which is not the current device")
    return i


def _ints(t, n: int, device: int, what: str):
    if t.dtype is not torch.int32 or t.shape != (n,) or t.stride(0) != 1 and n > 1 or t.get_device() != device:
        raise ValueError(f"{what} must be a contiguous int32 tensor of {n} elements on cuda:{device}")


def rope_table(n_positions: int, dims: int, theta: float = 10000.0, device="cuda"):
    """Cosine and sine of position * theta^(-2i/dims), computed in 64 bits: float32 [n_positions, dims / 2, 2]."""
    inv = float(theta) ** (-2.0 * torch.arange(dims // 2, dtype=torch.float64, device=device) / dims)
    angle = torch.arange(n_positions, dtype=torch.float64, device=device)[:, None] * inv
    return torch.stack([angle.cos(), angle.sin()], -1).float().contiguous()


class PagedCache:
    """Pools of keys and of values, [n_pages, n_kv_heads, page_size, d_head] (any strides with neighbouring elements in a row: a pool laid
    out [n_pages, page_size, n_kv_heads, d_head] is passed as its view `pool.transpose(1, 2)`).  fp32, bf16 or fp16; d_head 32, 64,
    96, 128 or 256; page_size a multiple of 16.  The tensors stay the caller's and are used in place.

    A block table is int32 [batch, max_pages]: position p of a sequence is row p % page_size of page table[sequence, p // page_size].
    Calls from several streams at a time are fine as far as the pools' contents allow it: every stream has a workspace of its own."""

    def __init__(self, k, v):
        if not torch.cuda.is_available():
            raise RuntimeError("xsm needs a CUDA device; there is no CPU path")
        self._h = C.c_void_p()
        self.lib = binding.load()
        _need(k.dim() == 4 and k.dtype in _DTYPES, "the pools must be [n_pages, n_kv_heads, page_size, d_head] of fp32, bf16 or fp16")
        _need(v.shape == k.shape and v.dtype == k.dtype and v.stride() == k.stride() and v.device == k.device, "both pools must be alike")
        _need(k.stride(3) == 1, "the elements of a row must be neighbours")
        self.device = _here(k)
        self.k, self.v, self.dtype = k, v, k.dtype
        self.n_pages, self.n_kv_heads, self.page_size, self.d_head = k.shape
        cfg = binding.KvConfig(*(s if n > 1 else k.shape[3] for s, n in zip((k.stride(0), k.stride(1), k.stride(2)), k.shape)), *k.shape,
                               _DTYPES[k.dtype])
        self._ws, self._ws_bytes = {}, {}
        _check(self.lib.xsm_kv_create(C.byref(cfg), k.data_ptr(), v.data_ptr(), C.byref(self._h)))

    def __del__(self):
        h, self._h = getattr(self, "_h", None), None
        if h:
            self.lib.xsm_kv_destroy(h)

    def _rows(self, x, what: str, heads=None):
        """Checks [batch, m, heads, d_head]; the strides."""
        if x.dim() != 4 or x.shape[3] != self.d_head or heads is not None and x.shape[2] != heads:
            raise ValueError(f"{what} must be [batch, m, {'n_heads' if heads is None else heads}, {self.d_head}], not {list(x.shape)}")
        if x.get_device() != self.device:
            raise ValueError(f"{what} must be on cuda:{self.device}")
        s = x.stride()
        if s[3] != 1:
            raise ValueError(f"the elements of a head of {what} must be neighbours")
        return s[:3]

    def _table(self, table, batch: int):
        if table.dtype is not torch.int32 or table.dim() != 2 or table.shape[0] != batch or table.get_device() != self.device or \
                table.shape[1] > 1 and table.stride(1) != 1:
            raise ValueError(f"the block table must be int32 [{batch}, max_pages] on cuda:{self.device}")
        return table.stride(0), table.shape[1]

    def append(self, k, v, block_table, starts, counts=None, q=None, rope=None, interleaved=False, out=None):
        """Writes k and v, [batch, m, n_kv_heads, d_head], to positions starts[b] + j (j < counts[b]) of every sequence; keys, and queries
        q [batch, m, n_heads, d_head], are rotated by `rope` (float32 [positions, dims / 2, 2], see rope_table).  Returns the rotated
        queries in `out` (a new tensor, or the one given; it may be q), or None without q."""
        device = _here(k)
        ks, vs = self._rows(k, "k", self.n_kv_heads), self._rows(v, "v", self.n_kv_heads)
        batch, m = k.shape[:2]
        if v.shape != k.shape or v.dtype is not k.dtype or k.dtype not in _DTYPES:
            raise ValueError("k and v must be alike, of fp32, bf16 or fp16")
        ld, pages = self._table(block_table, batch)
        _ints(starts, batch, self.device, "starts")
        if counts is not None:
            _ints(counts, batch, self.device, "counts")
        qs = os = (0, 0, 0)
        heads = positions = dims = 0
        if q is not None:
            qs, heads = self._rows(q, "q"), q.shape[2]
            if q.shape[:2] != k.shape[:2] or q.dtype is not k.dtype:
                raise ValueError("q must have the batch, the tokens and the type of k")
            if out is None:
                out = torch.empty(q.shape, dtype=q.dtype, device=q.device)
            os = self._rows(out, "out", heads)
            if out.shape != q.shape or out.dtype is not q.dtype:
                raise ValueError("out must have the shape and the type of q")
        else:
            out = None
        if rope is not None:
            if rope.dtype is not torch.float32 or rope.dim() != 3 or rope.shape[2] != 2 or not rope.is_contiguous() or rope.get_device() != self.device:
                raise ValueError(f"rope must be contiguous float32 [positions, dims / 2, 2] on cuda:{self.device}")
            positions, dims = rope.shape[0], 2 * rope.shape[1]
        _check(self.lib.xsm_kv_append(self._h, _APPEND.pack(
            _ptr(q), k.data_ptr(), v.data_ptr(), _ptr(out), block_table.data_ptr(), starts.data_ptr(), _ptr(counts), _ptr(rope),
            *qs, *ks, *vs, *os, ld, batch, m, heads, _DTYPES[k.dtype], pages, positions, dims, bool(interleaved)), _raw_stream(device)))
        return out

    def _workspace(self, stream: int, batch: int, m: int, heads: int):
        """Zeroed memory for the calls of a stream, kept from call to call."""
        need = self._ws_bytes.get((batch, m, heads))
        if need is None:
            need = self._ws_bytes[batch, m, heads] = max(16, self.lib.xsm_kv_attend_workspace(self._h, batch, m, heads))
        ws = self._ws.get(stream)
        if ws is None or ws.numel() < need:
            ws = torch.zeros(need, dtype=torch.uint8, device=self.k.device)
            if torch.cuda.is_current_stream_capturing():
                return ws          # the graph's own: zeroed whenever it is replayed
            self._ws[stream] = ws
        return ws

    def attend(self, q, block_table, lengths, counts=None, causal=True, window=0, scale=None, out=None, lse=None):
        """Attention of the newest tokens: q [batch, m, n_heads, d_head] over the first lengths[b] positions of every sequence, the new ones
        included.  Query j of n = counts[b] (m without counts) sees positions up to lengths[b] - n + j (all with causal=False), and
        of these the last `window` (0: all).  Returns (out, lse): out like q, lse float32 [batch, m, n_heads], the logarithm of the sum
        of exp(scale q.k), -inf where nothing is seen."""
        device = _here(q)
        qs = self._rows(q, "q")
        batch, m, heads, _ = q.shape
        if q.dtype not in _DTYPES:
            raise ValueError("q must be of fp32, bf16 or fp16")
        if q.requires_grad and torch.is_grad_enabled():
            raise ValueError("attend has no gradient: call it under torch.no_grad()")
        ld, pages = self._table(block_table, batch)
        _ints(lengths, batch, self.device, "lengths")
        if counts is not None:
            _ints(counts, batch, self.device, "counts")
        if out is None:
            out = torch.empty(q.shape, dtype=q.dtype, device=q.device)
        elif out.shape != q.shape or out.dtype is not q.dtype:
            raise ValueError("out must have the shape and the type of q")
        os = self._rows(out, "out")
        if lse is None:
            lse = torch.empty((batch, m, heads), dtype=torch.float32, device=q.device)
        elif lse.shape != (batch, m, heads) or lse.dtype is not torch.float32 or not lse.is_contiguous() or lse.get_device() != self.device:
            raise ValueError(f"lse must be contiguous float32 [{batch}, {m}, {heads}] on cuda:{self.device}")
        stream = _raw_stream(device)
        ws = self._workspace(stream, batch, m, heads)
        _check(self.lib.xsm_kv_attend(self._h, _ATTEND.pack(
            q.data_ptr(), out.data_ptr(), lse.data_ptr(), block_table.data_ptr(), lengths.data_ptr(), _ptr(counts), ws.data_ptr(),
            *qs, *os, ld, ws.numel(), batch, m, heads, _DTYPES[q.dtype], pages, bool(causal), window,
            self.d_head ** -0.5 if scale is None else scale), stream))
        return out, lse


def _check_logits(logits, tokens):
    device = _here(logits)
    if logits.dim() != 2 or logits.dtype not in _DTYPES or logits.stride(1) != 1 and logits.shape[1] > 1:
        raise ValueError("logits must be [rows, vocab] of fp32, bf16 or fp16 with neighbouring elements in a row")
    if tokens.dim() != 1 or tokens.shape[0] != logits.shape[0] or tokens.get_device() != device or \
            tokens.dtype is not torch.int64 and tokens.dtype is not torch.int32:
        raise ValueError(f"tokens must be int32 or int64 [{logits.shape[0]}] on cuda:{device}")
    return device


def _forward(logits, tokens, top, temperature):
    device = _check_logits(logits, tokens)
    rows, vocab = logits.shape
    logprob, entropy, lse = torch.empty((3, rows), dtype=torch.float32, device=logits.device).unbind(0)
    ids = alt = None
    if top > 0:
        ids = torch.empty((rows, top), dtype=torch.int32, device=logits.device)
        alt = torch.empty((rows, top), dtype=torch.float32, device=logits.device)
    _check(binding.load().xsm_token_logprobs(_LOGPROB.pack(
        logits.data_ptr(), tokens.data_ptr(), logprob.data_ptr(), entropy.data_ptr(), lse.data_ptr(), _ptr(ids), _ptr(alt),
        logits.stride(0), tokens.stride(0), rows, vocab, _DTYPES[logits.dtype], tokens.element_size(), top, temperature), _raw_stream(device)))
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
    missing.  out: a tensor like logits for the gradient, which may be the logits themselves."""
    device = _check_logits(logits, tokens)
    rows, vocab = logits.shape
    if out is None:
        out = torch.empty((rows, vocab), dtype=logits.dtype, device=logits.device)
    elif out.shape != logits.shape or out.dtype is not logits.dtype or out.get_device() != device or out.stride(1) != 1 and vocab > 1 or \
            out.stride(0) < vocab and rows > 1:
        raise ValueError("out must be like logits, with rows of their own")
    for t in (result.lse, result.entropy):
        if t.shape != (rows,) or t.dtype is not torch.float32 or t.get_device() != device or t.stride(0) != 1 and rows > 1:
            raise ValueError("result must be what token_logprobs returned for these logits")
    gl, gl_ld = _row_grad(grad_logprob, rows, device, "grad_logprob")
    ge, ge_ld = _row_grad(grad_entropy, rows, device, "grad_entropy")
    gs, gs_ld = _row_grad(grad_lse, rows, device, "grad_lse")
    top = ids = 0
    if grad_top is not None:
        ids = result.top_ids
        if ids is None or grad_top.shape != ids.shape or grad_top.dtype is not torch.float32 or not grad_top.is_contiguous() or \
                grad_top.get_device() != device or ids.dtype is not torch.int32 or not ids.is_contiguous() or ids.get_device() != device:
            raise ValueError("grad_top must be contiguous float32 [rows, top] beside the result's top_ids")
        top, ids = ids.shape[1], ids.data_ptr()
    _check(binding.load().xsm_token_logprobs_grad(_GRAD.pack(
        logits.data_ptr(), tokens.data_ptr(), result.lse.data_ptr(), result.entropy.data_ptr(), ids, gl, ge, gs, _ptr(grad_top),
        out.data_ptr(), logits.stride(0), tokens.stride(0), gl_ld, ge_ld, gs_ld, out.stride(0), rows, vocab, _DTYPES[logits.dtype],
        tokens.element_size(), top, temperature), _raw_stream(device)))
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
    largest logits, equal ones by the lower id first.  Differentiable by the logits."""
    if logits.requires_grad and torch.is_grad_enabled():
        return TokenLogprobs(*_TokenLogprobs.apply(logits, tokens, top, temperature))
    return _forward(logits, tokens, top, temperature)
