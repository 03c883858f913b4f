"""The model with the rotary positions in this library's kernel (own_rope): the
rotation and its gradient as the model's autograd sees them, packed documents, and
the step against the PyTorch form."""
import dataclasses
import math

import numpy as np
import pytest
import torch

import kv_reference as R
from gpu_util import DEV, log
from paper_2412_04787_amd import dqt, model_step as MS

pytestmark = pytest.mark.gpu


def test_rotation_and_its_gradient(lib):
    """Rotate's outputs and the gradients that autograd takes through it, views and
    broadcast gradients among its inputs, against float64."""
    log("model: rotation and its gradient")
    gen = torch.Generator().manual_seed(1)
    rotate = MS._OwnFns.get()[3]
    f = dqt.dqt_rope_freqs(64)
    rope = dqt.rope(64)
    T = 50
    wide = torch.randn((T, 6 * 64), generator=gen).to(torch.bfloat16).to(DEV).requires_grad_()
    x = wide.view(T, 6, 64)
    pos = torch.randint(0, 4000, (T,), generator=gen, dtype=torch.int32).to(DEV)
    q, k = rotate.apply(x[:, :4], x[:, 4:], pos, rope)
    g = torch.randn((T, 4, 64), generator=gen).to(torch.bfloat16)
    row = torch.randn((64,), generator=gen).to(torch.bfloat16)
    torch.autograd.backward((q, k), (g.to(DEV), row.to(DEV).expand(T, 2, 64)))
    torch.cuda.synchronize()
    at = pos.cpu().numpy()
    y, t = R.rotate(wide.detach().cpu().view(T, 6, 64), at, f, 64, False)
    got = torch.cat((q, k), 1).detach().double().cpu()
    assert ((got - y).abs() <= t + R.BF16 * y.abs() * (1 + R.BF16)).all()
    y, t = R.rotate(torch.cat((g, row.expand(T, 2, 64)), 1), at, f, 64, False, back=True)
    assert ((wide.grad.double().cpu().view(T, 6, 64) - y).abs() <= t + R.BF16 * y.abs() * (1 + R.BF16)).all()


def test_step_beside_the_pytorch_form(lib):
    """Same weights, same batch: the two forms' loss and dense gradients differ by the
    roundings of cosines to bf16 (2^-8 of each rotated value) and of what follows, as
    the operators' own test allows: 5 % of a gradient's norm for two layers."""
    log("model: own rotary positions beside PyTorch's")
    a, b = MS.DQTModel(MS.MODELS["tiny_rope"]), MS.DQTModel(MS.MODELS["tiny_ops"])
    tok, tgt = MS.synthetic_batch(MS.MODELS["tiny_rope"], 0)
    x, y = a.loss(tok, tgt), b.loss(tok, tgt)
    x.backward()
    y.backward()
    assert abs(float(x.detach()) - float(y.detach())) < 2e-3 * float(y.detach())
    for p, q in [(a.emb, b.emb), (a.head, b.head), (a.final_norm, b.final_norm)] + [z for n, m in zip(a.norms, b.norms) for z in zip(n, m)]:
        assert float((p.grad - q.grad).norm() / q.grad.norm()) < 0.05


def test_documents_stay_apart(lib):
    """A document's logits do not depend on the others nor on where it lies: positions
    count from its start."""
    cfg = MS.MODELS["tiny_rope"]
    model = MS.DQTModel(cfg)
    tok = MS.synthetic_batch(cfg, 1)[0].reshape(-1)
    s32 = lambda *x: torch.tensor(x, dtype=torch.int32, device=DEV)
    log("model: packed documents, own rotary positions")
    with torch.no_grad():
        a = model.logits(tok, s32(0, 100, 101, 256))
        b = model.logits(torch.cat([tok[101:], tok[:101]]), s32(0, 155, 255, 256))
    # (only the LM head's library product may sum in another order: one bf16 step)
    assert torch.allclose(b[:155].float(), a[101:].float(), rtol=2.0 ** -7, atol=2.0 ** -7 * float(a.float().abs().max()))


def test_trains(lib):
    cfg = MS.MODELS["tiny_rope"]
    log(f"training steps {cfg}")
    model = MS.DQTModel(cfg)
    losses = [float(model.train_step(*MS.synthetic_batch(cfg, s))) for s in range(3)]
    assert all(math.isfinite(v) for v in losses)
    changed, nonfinite = model.counters.tolist()
    assert changed > 0 and nonfinite == 0


def test_configuration_refusals():
    with pytest.raises(ValueError):
        dataclasses.replace(MS.MODELS["tiny"], own_rope=True)
