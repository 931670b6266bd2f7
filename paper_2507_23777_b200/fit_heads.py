"""Offline weight preparation: fit the decoding heads of a synthetic model to its own backbone.

The synthetic configurations draw every weight independently, so their decoding heads know nothing about the
backbone and almost no draft is ever accepted.  The method assumes heads that were distilled from the backbone
(Sec. 4.3, Backbone Distillation Training).  This script does the first stage of that training on a synthetic
model: the backbone stays frozen, it generates token sequences for a set of meshes (through the library's own
plain one-token-per-step path), and head d is trained with the cross-entropy of Eq. 4 to predict token
s + d + 1 from the backbone's final hidden state of position s, the heads weighted by w(d) = 0.8^d (Eq. 5 and
the implementation details of Sec. 5.1).  The second stage (LoRA on the backbone) is not done: the backbone
and its K = 0 baseline stay exactly the configured ones.

Every head starts as a copy of the LM head with a zero residual block (a head that repeats the backbone's
own next-token guess) and is fine-tuned with AdamW; the checkpoint with the lowest loss on held-out meshes is
kept, the starting point included.  The result is a weight buffer in the library's layout that differs from the
input only in the heads.

PyTorch does the training arithmetic here (a forward pass of the backbone over whole sequences, and the
optimiser).  None of this is on the decoding path: the library never imports this module.

    python -m paper_2507_23777_b200.fit_heads --config 2            # fit, then decode with K heads and with K = 0
"""
from __future__ import annotations

import argparse
import json
import time

import numpy as np

from . import inputs


def _views(cfg: dict, Wf):
    offs = inputs.weight_offsets(cfg)

    def W(name):
        o, shp = offs[name]
        n = int(np.prod(shp))
        return Wf[o:o + n].view(*shp)
    return W


def _need_bf16(cfg: dict):
    if cfg["dtype"] != 1:
        raise ValueError("the library's products are of 16-bit weights: the model must be a bf16 one")


def backbone_hidden(cfg: dict, Wf, tokens: np.ndarray, cond: np.ndarray, device="cuda", library_products=False):
    """Final hidden states g_s = RMSNorm_f(h^N_s) of a whole token sequence under the causal mask (Eq. 1; block
    order and norms as in Sec. 4.1 and the library header): tensor [len(tokens), d_model] on `device`.
    Wf: all weights as one fp32 tensor on `device`.  library_products: the gated feed-forward parts by the library's operator (ops.gated_feed_forward, a GPU is needed), on
    activations and weights that are rounded to bf16; the model must be a bf16 one."""
    import torch
    import torch.nn.functional as F
    if library_products:
        _need_bf16(cfg)
    W = _views(cfg, Wf)
    L, d, H, dh = cfg["n_layers"], cfg["d_model"], cfg["n_heads"], cfg["d_head"]
    n, half = len(tokens), dh // 2
    x = torch.as_tensor(np.asarray(tokens, dtype=np.int64), device=device)
    c = torch.as_tensor(np.asarray(cond, dtype=np.float32), device=device)

    def rms(v, g):
        return v * torch.rsqrt((v * v).mean(-1, keepdim=True) + cfg["rms_eps"]) * g

    inv = cfg["rope_theta"] ** (-2.0 * torch.arange(half, device=device, dtype=torch.float64) / dh)
    ang = torch.arange(n, device=device, dtype=torch.float64)[:, None] * inv[None, :]
    cs, sn = ang.cos().float()[:, None, :], ang.sin().float()[:, None, :]

    def rope(v):           # [n, H, dh], pairs (i, i + dh/2)
        a, b = v[..., :half], v[..., half:]
        return torch.cat([a * cs - b * sn, a * sn + b * cs], -1)

    def attend(q, k, v, causal):
        o = F.scaled_dot_product_attention(q.transpose(0, 1)[None], k.transpose(0, 1)[None], v.transpose(0, 1)[None],
                                           is_causal=causal)[0]
        return o.transpose(0, 1).reshape(q.shape[0], d)

    with torch.no_grad():
        h = W("E")[x]
        for l in range(L):
            p = f"l{l}."
            u = rms(h, W(p + "g1"))
            q, k = rope((u @ W(p + "Wq").T).view(n, H, dh)), rope((u @ W(p + "Wk").T).view(n, H, dh))
            h = h + attend(q, k, (u @ W(p + "Wv").T).view(n, H, dh), True) @ W(p + "Wo").T
            u = rms(h, W(p + "g2"))
            kc, vc = (c @ W(p + "Wkc").T).view(-1, H, dh), (c @ W(p + "Wvc").T).view(-1, H, dh)
            h = h + attend((u @ W(p + "Wqc").T).view(n, H, dh), kc, vc, False) @ W(p + "Woc").T
            u = rms(h, W(p + "g3"))
            if library_products:
                from . import ops
                y = ops.gated_feed_forward(u.bfloat16(), W(p + "Wgate").bfloat16(), W(p + "Wup").bfloat16()).float()
            else:
                y = F.silu(u @ W(p + "Wgate").T) * (u @ W(p + "Wup").T)
            h = h + y @ W(p + "Wdown").T
        return rms(h, W("gf"))


def fit_from_corpus(cfg: dict, weights: np.ndarray, seqs, conds, iters=300, lr=2e-5, eval_every=25, holdout=0.125,
                    batch=4096, device="cuda", seed=0, library_loss=False, library_products=False):
    """seqs[i]: tokens x_0.. of mesh i (x_0 = BOS) generated by the backbone, conds[i]: its condition [C, d_cond].
    library_loss: cross-entropy and its gradient by the library's operator (ops.token_logprobs, a GPU is needed) instead of torch's.  library_products: the backbone's gated
    feed-forward parts, and the loss straight from the heads' hidden states without logits (ops.linear_logprobs), by the library's operators in bf16 (bf16 models).
    Returns (weights with fitted heads, report)."""
    if library_products:
        _need_bf16(cfg)
    import torch
    import torch.nn.functional as F
    K, d, V = cfg["n_draft"], cfg["d_model"], cfg["vocab"]
    assert K >= 1 and cfg["head_hidden"] == d
    torch.manual_seed(seed)
    Wf = torch.from_numpy(inputs.weights_as_f32(cfg, weights).astype(np.float32, copy=True)).to(device)
    W = _views(cfg, Wf)
    G = [backbone_hidden(cfg, Wf, s[:-1], c, device, library_products) for s, c in zip(seqs, conds)]
    X = [torch.as_tensor(np.asarray(s, dtype=np.int64), device=device) for s in seqs]

    def dataset(idx):       # input g_s; target of head d (1..K): x_{s+d+1}
        gs, ys = [], []
        for j in idx:
            n = len(G[j]) - K - 1
            if n > 0:
                gs.append(G[j][:n])
                ys.append(torch.stack([X[j][1 + dd:1 + dd + n] for dd in range(1, K + 1)], 1))
        return torch.cat(gs), torch.cat(ys)

    n_hold = max(1, int(round(len(seqs) * holdout)))
    g_te, y_te = dataset(range(n_hold))
    g_tr, y_tr = dataset(range(n_hold, len(seqs)))
    W1 = [torch.zeros(d, d, device=device, requires_grad=True) for _ in range(K)]
    Wo = [W("W0").clone().requires_grad_(True) for _ in range(K)]
    opt = torch.optim.AdamW(W1 + Wo, lr=lr, weight_decay=0.0)

    def states(g, i):
        return g + F.silu(g @ W1[i].T)

    def head(g, i):
        return states(g, i) @ Wo[i].T

    if library_loss:
        from . import ops

        def entropy_of(z, t):
            return -ops.token_logprobs(z, t).logprob.mean()
    else:
        entropy_of = F.cross_entropy

    if library_products:
        from . import ops

        def loss_of_head(g, i, t):
            return -ops.linear_logprobs(states(g, i).bfloat16(), Wo[i].bfloat16(), t).logprob.mean()
    else:
        def loss_of_head(g, i, t):
            return entropy_of(head(g, i), t)

    def loss_of(g, y):      # Eq. 5 with w(d) = 0.8^d
        return sum(0.8 ** (i + 1) * loss_of_head(g, i, y[:, i]) for i in range(K))

    curve, best, best_state, best_it = [], None, None, 0
    for it in range(iters + 1):
        if it % eval_every == 0 or it == iters:
            with torch.no_grad():
                hl = float(loss_of(g_te, y_te))
                acc = [float((head(g_te, i).argmax(-1) == y_te[:, i]).float().mean()) for i in range(K)]
            curve.append({"iteration": it, "held_out_loss": hl, "held_out_top1": acc})
            if best is None or hl < best:
                best, best_it, best_state = hl, it, [w.detach().clone() for w in W1 + Wo]
        if it == iters:
            break
        idx = torch.randint(0, len(g_tr), (min(batch, len(g_tr)),), device=device)
        loss = loss_of(g_tr[idx], y_tr[idx])
        opt.zero_grad()
        loss.backward()
        opt.step()
    if library_products:
        ops.check()
    out = inputs.weights_as_f32(cfg, weights).astype(np.float32, copy=True)
    offs = inputs.weight_offsets(cfg)
    for i in range(K):
        o, _ = offs[f"h{i + 1}.W1"]
        out[o:o + d * d] = best_state[i].cpu().numpy().ravel()
        o, _ = offs[f"h{i + 1}.Wout"]
        out[o:o + V * d] = best_state[K + i].cpu().numpy().ravel()
    fitted = inputs.f32_to_bf16_bits(out) if cfg["dtype"] == 1 else out
    report = {"meshes": len(seqs), "held_out_meshes": n_hold, "training_positions": int(len(g_tr)), "iterations": iters,
              "kept_iteration": best_it, "held_out_loss_start": curve[0]["held_out_loss"], "held_out_loss_kept": best,
              "lr": lr, "curve": curve}
    return fitted, report


def corpus(cfg: dict, weights: np.ndarray, n_meshes: int, n_tokens: int, seed0: int = 5000):
    """Token sequences of `n_meshes` meshes (conditions and Philox streams seeded seed0, seed0 + 1, ...) from the
    library's K = 0 path under the configuration's own verification and sampling rule."""
    from . import binding
    cfg0 = dict(cfg, n_draft=0)
    w0 = np.ascontiguousarray(weights[:inputs.n_weight_elements(cfg0)])
    ctx = binding.Context(cfg0, w0, max_batch=1)
    seqs, conds = [], []
    for i in range(n_meshes):
        c = dict(cfg0, seed=seed0 + i)
        cond = inputs.make_cond(c, 1)
        ctx.prefill(cond, [cfg["bos_id"]], binding.decode_config(c))
        toks, _, _ = ctx.generate(n_tokens)
        seqs.append(np.concatenate([[cfg["bos_id"]], toks[0]]).astype(np.int64))
        conds.append(cond[0])
    ctx.xsm_destroy()
    return seqs, conds


def fit(cfg: dict, weights: np.ndarray, n_meshes=96, n_tokens=512, seed0=5000, **kw):
    t0 = time.time()
    seqs, conds = corpus(cfg, weights, n_meshes, n_tokens, seed0)
    t1 = time.time()
    fitted, report = fit_from_corpus(cfg, weights, seqs, conds, **kw)
    report.update({"tokens_per_mesh": n_tokens, "corpus_seconds": t1 - t0, "fit_seconds": time.time() - t1,
                   "corpus_seed0": seed0})
    return fitted, report


def main():
    from . import binding, build
    ap = argparse.ArgumentParser()
    ap.add_argument("--config", type=int, default=2)
    ap.add_argument("--meshes", type=int, default=96)
    ap.add_argument("--tokens", type=int, default=512, help="tokens per training mesh")
    ap.add_argument("--iters", type=int, default=300)
    ap.add_argument("--lr", type=float, default=2e-5)
    ap.add_argument("--library-loss", action="store_true", help="cross-entropy and its gradient by the library's operator")
    ap.add_argument("--library-products", action="store_true", help="gated feed-forward parts, and the loss without logits, by the library's operators (bf16 models)")
    ap.add_argument("--eval-tokens", type=int, default=4096)
    ap.add_argument("--eval-seeds", type=int, nargs="*", default=None, help="mesh seeds to decode (default: the configuration's)")
    args = ap.parse_args()
    build.build()
    cfg = inputs.config(args.config)
    w = inputs.make_weights(cfg)
    fitted, report = fit(cfg, w, args.meshes, args.tokens, iters=args.iters, lr=args.lr, library_loss=args.library_loss, library_products=args.library_products)
    report.pop("curve")
    print(json.dumps({"fit": report}))
    cfg0 = dict(cfg, n_draft=0)
    runs = [("configured heads", cfg, w), ("fitted heads", cfg, fitted),
            ("K = 0", cfg0, np.ascontiguousarray(w[:inputs.n_weight_elements(cfg0)]))]
    for seed in (args.eval_seeds or [cfg["seed"]]):
        for name, c, ww in runs:
            c = dict(c, seed=seed)
            ctx = binding.Context(c, ww, max_batch=1)
            cond = inputs.make_cond(c, 1)
            for _ in range(2):          # the second pass is the timed one
                ctx.prefill(cond, [c["bos_id"]], binding.decode_config(c))
                _, _, st = ctx.generate(args.eval_tokens)
            print(json.dumps({"mesh_seed": seed, "heads": name, "scr": st.scr, "tokens_per_s": args.eval_tokens / st.wall_ms * 1e3,
                              "us_per_step": st.wall_ms * 1e3 / st.steps, "accept_hist": list(st.accept_hist)[:c["n_draft"] + 1]}))
            ctx.xsm_destroy()


if __name__ == "__main__":
    main()
