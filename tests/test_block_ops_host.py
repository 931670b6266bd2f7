"""The torch side of the operators on a caller's own activations and weights, and the paths that call them, where no device is needed."""
import numpy as np
import pytest
import torch

from paper_2507_23777_b200 import binding, build, ops


@pytest.fixture(scope="module")
def lib():
    build.build()
    return binding.load()


def test_sizes_of_workspaces_are_each_devices_own(monkeypatch):
    """Devices of unequal numbers of SMs need workspaces of unequal sizes."""
    class Lib:
        current = 0

        def xsm_linear_logprobs_workspace(self, rows, vocab, d):
            return 1000 + self.current
    fake = Lib()
    monkeypatch.setattr(ops, "_sizes", {})
    monkeypatch.setattr(ops.binding, "load", lambda: fake)
    for fake.current in (0, 3, 0, 3):
        assert ops._size_of("xsm_linear_logprobs_workspace", fake.current, 4, 100, 64) == 1000 + fake.current


def test_threads_share_a_devices_status_word(monkeypatch):
    """Another thread makes the word while this one does: both use the first, which is the one that check reads."""
    theirs = torch.zeros(16, dtype=torch.uint8)
    words = {}

    def zeros(*args, **kw):
        words[2] = theirs
        return torch.ones(16, dtype=torch.uint8)
    monkeypatch.setattr(ops, "_status_words", words)
    monkeypatch.setattr(ops.torch, "zeros", zeros)
    assert ops._status(2, 0) == theirs.data_ptr() and words[2] is theirs


@pytest.mark.parametrize("temperature", [4.2e-39, 3e-39])
def test_temperatures_whose_factor_is_infinite_are_refused(lib, temperature):
    """log2(e) / T is what logits are multiplied by: infinite, it makes NaN of every zero.  (1 / T is finite here.)"""
    A = 4096
    args = ops._LINEAR.pack(*8 * [A], 64, 64, 1, 1 << 30, 4, 100, 64, 1, 8, temperature)
    assert lib.xsm_linear_logprobs(args, None) == binding.XSM_ERR_INVALID_ARG and b"temperature" in lib.xsm_last_error(None)
    args = ops._LINEAR_GRAD.pack(*11 * [A], 64, 64, 1, 1, 1, 64, 64, 1 << 30, 4, 100, 64, 1, 8, temperature)
    assert lib.xsm_linear_logprobs_grad(args, None) == binding.XSM_ERR_INVALID_ARG and b"temperature" in lib.xsm_last_error(None)


def test_heads_of_fp32_models_are_not_fitted_in_bf16():
    """As scoring refuses it: the library's products would round weights that the model holds in 32 bits."""
    from paper_2507_23777_b200 import fit_heads, inputs
    cfg = inputs.config(0)
    w = inputs.make_weights(cfg)
    seqs, conds = [np.arange(4)] * 2, list(inputs.make_cond(cfg, 2))
    with pytest.raises(ValueError, match="bf16"):
        fit_heads.fit_from_corpus(cfg, w, seqs, conds, iters=0, device="cpu", library_products=True)
    with pytest.raises(ValueError, match="bf16"):
        fit_heads.backbone_hidden(cfg, torch.from_numpy(inputs.weights_as_f32(cfg, w).astype(np.float32)), seqs[0], conds[0], "cpu", library_products=True)
