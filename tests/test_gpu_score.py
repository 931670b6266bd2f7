"""Scoring of given meshes (score.py) against a whole-sequence forward pass, and the heads' loss through the library's operator."""
import numpy as np
import pytest
import torch

from conftest import gpu_cfg
from paper_2507_23777_b200 import inputs

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def score():
    assert torch.cuda.is_available(), "this test needs a B200"
    from paper_2507_23777_b200 import build, score
    build.build()
    return score


@pytest.mark.parametrize("dtype,bound", [(0, 2e-4), (1, 2e-2)])
@pytest.mark.parametrize("batch,n", [(1, 2), (2, 17), (3, 90)])
def test_scores_equal_those_of_a_whole_sequence(score, dtype, bound, batch, n):
    """The library's own bounds on logits, fp32 2e-4 and bf16 models (fp16 caches) 2e-2, twice: a logit and the sum over all."""
    from paper_2507_23777_b200 import fit_heads
    cfg = gpu_cfg(dtype=dtype, sigma=0.08, seed=3, batch=batch)
    w = inputs.make_weights(cfg, random_gains=True)
    cond = inputs.make_cond(cfg, batch)
    tokens = np.random.default_rng(n).integers(1, cfg["vocab"], (batch, n))
    tokens[:, 0] = cfg["bos_id"]
    s = score.Scorer(cfg, w, batch, n)
    r = s.score(cond, tokens, top=3)
    flat = torch.from_numpy(inputs.weights_as_f32(cfg, w).astype(np.float32, copy=True)).cuda()
    for b in range(batch):
        g = fit_heads.backbone_hidden(cfg, flat, tokens[b, :-1], cond[b])
        z = (g @ s.W("W0").T).double()
        logp = torch.log_softmax(z, -1)
        want = logp.gather(1, torch.as_tensor(tokens[b, 1:], device="cuda")[:, None])[:, 0]
        assert float((r.logprob[b].double() - want).abs().max()) < 2 * bound
        assert float((r.entropy[b].double() - torch.special.entr(logp.exp()).sum(-1)).abs().max()) < 2 * bound * np.log(cfg["vocab"])
        best = z.topk(3, -1).values
        clear = (best[:, :2] - best[:, 1:]).min(-1).values > 2 * bound
        assert torch.equal(r.top_ids[b][clear][:, :2].long(), z.topk(2, -1).indices[clear])


def test_greedy_meshes_are_their_own_best_alternatives(score):
    """Tokens decoded by the library with strict greedy verification are the best alternative wherever the two best are not close."""
    from paper_2507_23777_b200 import binding
    cfg = gpu_cfg(dtype=1, sigma=0.08, seed=5, max_seq_len=200)
    w, cond = inputs.make_weights(cfg, random_gains=True), inputs.make_cond(cfg, 1)
    ctx = binding.Context(cfg, w, max_batch=1)
    ctx.prefill(cond, [cfg["bos_id"]], binding.decode_config(cfg))
    mesh = np.concatenate([[cfg["bos_id"]], ctx.generate(150)[0][0]])
    ctx.xsm_destroy()
    r = score.Scorer(cfg, w, 1, 150).score(cond, mesh[None], top=2)
    clear = r.top_logprobs[0, :, 0] - r.top_logprobs[0, :, 1] > 4e-2
    assert int(clear.sum()) > 75
    assert torch.equal(r.top_ids[0, :, 0][clear].long(), torch.as_tensor(mesh[1:], device="cuda")[clear])


def test_refusals(score):
    cfg = gpu_cfg(dtype=1)
    s = score.Scorer(cfg, inputs.make_weights(cfg), 2, 20)
    cond = inputs.make_cond(cfg, 2)
    for shape in ((1, 5), (2, 1), (2, 22)):
        with pytest.raises(ValueError):
            s.score(cond, np.zeros(shape, dtype=np.int64))


def test_heads_fitted_with_the_operators_loss(score):
    """The same training with torch's cross-entropy and with the library's: losses within the rounding of a few steps of fp32 training."""
    from paper_2507_23777_b200 import fit_heads
    cfg = gpu_cfg(dtype=0, sigma=0.1, seed=11, n_draft=2)
    w = inputs.make_weights(cfg)
    rng = np.random.default_rng(0)
    seqs = [np.concatenate([[0], rng.integers(0, cfg["vocab"], 60)]) for _ in range(4)]
    conds = list(inputs.make_cond(cfg, 4))
    runs = [fit_heads.fit_from_corpus(cfg, w, seqs, conds, iters=12, lr=1e-3, eval_every=4, library_loss=lib)[1] for lib in (False, True)]
    a, b = ([c["held_out_loss"] for c in r["curve"]] for r in runs)
    assert len(a) == 4 and a[0] != a[-1]
    assert np.allclose(a, b, rtol=1e-4)


def test_tokens_outside_the_vocabulary_are_refused(score):
    """On the host, before anything is looked up by them; the scorer is as good as before."""
    cfg = gpu_cfg(dtype=1)
    s = score.Scorer(cfg, inputs.make_weights(cfg), 1, 20)
    cond = inputs.make_cond(cfg, 1)
    good = np.array([[cfg["bos_id"], 3, 7, cfg["vocab"] - 1]])
    want = s.score(cond, good).logprob
    for bad in (-1, cfg["vocab"], 2 ** 40, -(2 ** 40)):
        for place in (0, 2, 3):
            tokens = good.copy()
            tokens[0, place] = bad
            with pytest.raises(ValueError):
                s.score(cond, tokens)
    with pytest.raises(ValueError):
        s.score(cond, good + 0.5)
    assert torch.equal(s.score(cond, good).logprob, want)


def test_logits_behind_tokens_outside_the_vocabulary_are_nan(score):
    cfg = gpu_cfg(dtype=0)
    s = score.Scorer(cfg, inputs.make_weights(cfg), 1, 20)
    s.condition(inputs.make_cond(cfg, 1))
    tokens = torch.tensor([[cfg["bos_id"], 3, cfg["vocab"], 4]], device="cuda")
    z = s.logits(tokens, 0)
    s.condition(inputs.make_cond(cfg, 1))
    assert torch.equal(z[:, :2], s.logits(tokens.clamp(max=cfg["vocab"] - 1), 0)[:, :2]) and z[:, 2:].isnan().all()
    assert s.logits(torch.tensor([[-1]], device="cuda"), 4).isnan().all()


@pytest.mark.parametrize("which", ["cache", "cond_cache"])
def test_scores_of_an_attention_that_gave_up_are_not_returned(score, which):
    from paper_2507_23777_b200 import binding
    cfg = gpu_cfg(dtype=1)
    s = score.Scorer(cfg, inputs.make_weights(cfg), 1, 40)
    cond, tokens = inputs.make_cond(cfg, 1), np.arange(40)[None]
    want = s.score(cond, tokens).logprob
    some = getattr(s, which)
    for c in some:
        c.lib.xsm_debug_kv_waits(c._h, 20, 1)
    with pytest.raises(binding.XsmError) as e:
        s.score(cond, tokens)
    assert e.value.status == binding.XSM_ERR_TIMEOUT
    for c in some:
        c.lib.xsm_debug_kv_waits(c._h, 0, 0)
    assert torch.equal(s.score(cond, tokens).logprob, want)
