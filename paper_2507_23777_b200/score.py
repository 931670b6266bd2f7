"""Scores given meshes: the log probability of every token of a sequence under a backbone, its entropy and the best alternatives.

The sequences go through the backbone of the library's weight layout (include/xsm.h) a window of tokens at a time, as a decoder with
projections of its own would do it: torch multiplies, the library's operators (ops.py) append the window's keys and values to the pages,
attend the window over them and over the condition's, and turn the logits into log probabilities.  A block of another kind (grouped heads,
a sliding window, other norms) needs other lines here and nothing else.

    python -m paper_2507_23777_b200.score --config 1 --tokens 256      # decode a mesh with the library, then score it
"""
from __future__ import annotations

import argparse
import json

import numpy as np
import torch
import torch.nn.functional as F

from . import binding, inputs, ops

WINDOW = 16          # tokens of a sequence that go through the backbone at a time: what xsm_kv_attend takes


class Scorer:
    """A backbone's weights on the GPU and the paged caches of `batch` sequences of up to max_tokens tokens."""

    def __init__(self, cfg: dict, weights: np.ndarray, batch: int = 1, max_tokens: int | None = None):
        self.cfg, self.batch, dev = cfg, batch, "cuda"
        flat = torch.from_numpy(inputs.weights_as_f32(cfg, weights).astype(np.float32, copy=True)).to(dev)
        offs = inputs.weight_offsets(cfg)
        self.W = lambda name: flat[offs[name][0]:offs[name][0] + int(np.prod(offs[name][1]))].view(*offs[name][1])
        L, H, P, dh, C = (cfg[n] for n in ("n_layers", "n_heads", "page_size", "d_head", "n_cond"))
        self.max_tokens = max_tokens or cfg["max_seq_len"]
        kind = torch.float16 if cfg["dtype"] == 1 else torch.float32       # as the library keeps its own models' caches

        def caches(positions):
            pages = -(-positions // P)
            table = torch.arange(batch * pages, dtype=torch.int32, device=dev).view(batch, pages)
            return table, [ops.PagedCache(*(torch.empty((batch * pages, H, P, dh), dtype=kind, device=dev) for _ in range(2))) for _ in range(L)]
        self.table, self.cache = caches(self.max_tokens)
        self.cond_table, self.cond_cache = caches(C)
        self.rope = ops.rope_table(self.max_tokens, dh, cfg["rope_theta"], dev)
        self.cond_length = torch.full((batch,), C, dtype=torch.int32, device=dev)

    def _norm(self, x, gain):
        return x * torch.rsqrt((x * x).mean(-1, keepdim=True) + self.cfg["rms_eps"]) * self.W(gain)

    def _heads(self, x, name):
        return (x @ self.W(name).T).view(self.batch, x.shape[1], self.cfg["n_heads"], self.cfg["d_head"])

    @torch.no_grad()
    def condition(self, cond):
        """Keys and values of the condition [batch, n_cond, d_cond], once for a mesh."""
        c = torch.as_tensor(cond, dtype=torch.float32, device="cuda")
        zero = torch.zeros(self.batch, dtype=torch.int32, device="cuda")
        for l, cache in enumerate(self.cond_cache):
            cache.append(self._heads(c, f"l{l}.Wkc"), self._heads(c, f"l{l}.Wvc"), self.cond_table, zero)

    @torch.no_grad()
    def logits(self, tokens, start: int):
        """Logits behind tokens [batch, m] at positions start, start + 1, ...: [batch, m, vocab]; the caches hold the positions before.  Behind a token
        outside the vocabulary they are NaN."""
        m, vocab = tokens.shape[1], self.cfg["vocab"]
        at = torch.full((self.batch,), start, dtype=torch.int32, device="cuda")
        h = self.W("E")[tokens.clamp(0, vocab - 1)].masked_fill(((tokens < 0) | (tokens >= vocab))[..., None], float("nan"))
        for l in range(self.cfg["n_layers"]):
            p, cache, cond = f"l{l}.", self.cache[l], self.cond_cache[l]
            u = self._norm(h, p + "g1")
            q = cache.append(self._heads(u, p + "Wk"), self._heads(u, p + "Wv"), self.table, at, q=self._heads(u, p + "Wq"), rope=self.rope)
            h = h + cache.attend(q, self.table, at + m)[0].flatten(2) @ self.W(p + "Wo").T
            q = self._heads(self._norm(h, p + "g2"), p + "Wqc")
            h = h + cond.attend(q, self.cond_table, self.cond_length, causal=False)[0].flatten(2) @ self.W(p + "Woc").T
            u = self._norm(h, p + "g3")
            h = h + (F.silu(u @ self.W(p + "Wgate").T) * (u @ self.W(p + "Wup").T)) @ self.W(p + "Wdown").T
        return self._norm(h, "gf") @ self.W("W0").T

    @torch.no_grad()
    def score(self, cond, tokens, top: int = 0, temperature: float = 1.0) -> ops.TokenLogprobs:
        """tokens [batch, n], x_0 = BOS: (logprob, entropy, lse) [batch, n - 1] of x_1 .. x_{n-1}, and with `top` the best ids and their log
        probabilities [batch, n - 1, top] at every place.  Waits for the device; an XsmError where a wait of the attention ran out."""
        tokens = np.asarray(tokens)
        if tokens.ndim != 2 or tokens.shape[0] != self.batch or not 2 <= tokens.shape[1] <= self.max_tokens + 1:
            raise ValueError(f"tokens must be [{self.batch}, 2 to {self.max_tokens + 1}]")
        if tokens.dtype.kind not in "iuf" or (tokens != np.floor(tokens)).any() or tokens.min() < 0 or tokens.max() >= self.cfg["vocab"]:
            raise ValueError(f"tokens must be whole numbers in [0, {self.cfg['vocab']})")
        x = torch.as_tensor(tokens.astype(np.int64), device="cuda")
        self.condition(cond)
        parts = []
        for a in range(0, x.shape[1] - 1, WINDOW):
            m = min(WINDOW, x.shape[1] - 1 - a)
            z = self.logits(x[:, a:a + m], a).flatten(0, 1)
            r = ops.token_logprobs(z, x[:, a + 1:a + 1 + m].flatten(), top=top, temperature=temperature)
            parts.append([None if t is None else t.view(self.batch, m, *t.shape[1:]) for t in r])
        gave_up = None
        for cache in self.cache + self.cond_cache:          # (all of them: none is to tell the next score of this one's)
            try:
                cache.check()
            except binding.XsmError as e:
                gave_up = e
        if gave_up is not None:
            raise gave_up
        return ops.TokenLogprobs(*(None if p[0] is None else torch.cat(p, 1) for p in zip(*parts)))


def main():
    from . import build
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--config", type=int, default=1)
    ap.add_argument("--tokens", type=int, default=256)
    ap.add_argument("--top", type=int, default=5)
    args = ap.parse_args()
    build.build()
    cfg = inputs.config(args.config, batch=1)
    w, cond = inputs.make_weights(cfg), inputs.make_cond(cfg, 1)
    ctx = binding.Context(cfg, w, max_batch=1)
    ctx.prefill(cond, [cfg["bos_id"]], binding.decode_config(cfg))
    mesh = np.concatenate([[cfg["bos_id"]], ctx.generate(args.tokens)[0][0]])
    ctx.xsm_destroy()
    r = Scorer(cfg, w, 1, args.tokens).score(cond, mesh[None], top=args.top)
    place = (r.top_ids[0] == torch.as_tensor(mesh[1:], device="cuda")[:, None]).any(-1)
    print(json.dumps({"config": cfg["name"], "tokens": args.tokens, "log_probability": float(r.logprob.sum()), "perplexity": float((-r.logprob.mean()).exp()),
                      "mean_entropy": float(r.entropy.mean()), f"share_in_best_{args.top}": float(place.float().mean())}))


if __name__ == "__main__":
    main()
