"""Host-side pieces of the model step: flop accounting against the closed
forms, the device packing of ternary codes against the oracle's, and the
targets that the loss and the score hand to the library."""
import ctypes

import numpy as np
import pytest
import torch

from oracle import dqt_oracle as O
from paper_2412_04787_amd import dqt, model_step as MS


def test_step_flops_closed_forms():
    c = MS.MODELS["llama24_h2048"]
    f = c.step_flops()
    T, H, F, L = 8 * 2048, 2048, 5632, 24
    assert c.dqt_weights == L * (4 * H * H + 3 * H * F) == 1_233_125_376
    assert f["dqt_linears"] == 6 * T * c.dqt_weights
    assert f["lm_head"] == 6 * T * 32000 * H
    # causal attention: Q K^T and P V over half of the S x S scores, forward
    # (2 products x 2 flop x S^2 / 2 x H per sequence) and a backward of twice that
    assert f["attention"] == 3 * (2 * 2 * 8 * 2048 * 2048 * H // 2) * L
    assert abs(f["total"] / 1e12 - 137.56) < 0.01


def test_pack_ternary_matches_oracle():
    rng = np.random.default_rng(3)
    q = rng.integers(-1, 2, size=(48, 64)).astype(np.int8)
    got = MS._pack_ternary_dev(torch.from_numpy(q)).numpy()
    assert np.array_equal(got, O.pack_ternary(q))


class _Library:
    """Stands for the library: keeps the targets that its calls would read."""

    def __init__(self, rows):
        self.rows, self.read = rows, []

    def _targets(self, address):
        self.read.append(list((ctypes.c_int64 * self.rows).from_address(address)))
        return dqt.DQT_OK

    def dqt_logprob_workspace(self, M, V, top_k):
        return 0

    def dqt_logprob_fwd(self, X, x_t, M, V, stride, targets, *rest):
        return self._targets(targets)

    def dqt_logprob_bwd(self, X, x_t, M, V, stride, targets, *rest):
        return self._targets(targets)


@pytest.fixture
def headless(monkeypatch):
    """A model with own_ops whose logits are given, in host memory."""
    cfg = MS.MODELS["tiny_ops"]
    lib = _Library(cfg.tokens)
    monkeypatch.setattr(dqt, "load", lambda: lib)
    monkeypatch.setattr(dqt, "_here", lambda *t: -1)
    monkeypatch.setattr(dqt, "_stream", lambda stream=None: None)
    model = MS.DQTModel.__new__(MS.DQTModel)
    model.cfg, model._ws = cfg, None
    x = torch.zeros((cfg.tokens, cfg.vocab), requires_grad=True)
    model.logits = lambda tokens, starts=None: x * 1.0
    return model, lib


@pytest.mark.parametrize("form", ["plain", "interleaved", "transposed", "one row"])
def test_targets_of_any_strides(headless, form):
    """The library reads targets as consecutive int64: loss, gradient and score
    of a strided tensor are those of its values."""
    model, lib = headless
    B, S = model.cfg.batch, model.cfg.seq
    ids = torch.arange(B * S * 2, dtype=torch.int64).reshape(B, S, 2) % model.cfg.vocab
    t = {"plain": ids[..., 1].contiguous(), "interleaved": ids[..., 1],
         "transposed": ids[..., 1].t().contiguous().t(), "one row": ids[:1, :1, 0].expand(B, S)}[form]
    want = t.flatten().tolist()
    loss = model.loss(None, t)
    loss.backward()
    model.score(None, t)
    assert lib.read == [want] * 3


def test_targets_of_another_type_or_number_are_refused(headless):
    model, lib = headless
    t = torch.zeros((model.cfg.batch, model.cfg.seq), dtype=torch.int64)
    for bad in (t.int(), t[:, 1:], t.float()):
        for call in (model.loss, model.score):
            with pytest.raises(ValueError):
                call(None, bad)
    assert lib.read == []
