"""The model with attention, SwiGLU and loss in this library's kernels
(own_ops): against the same model in PyTorch, packed documents, scoring, and
all of the operators' calls captured into a graph."""
import dataclasses
import math

import pytest
import torch

import op_reference as R
from gpu_util import DEV, log
from paper_2412_04787_amd import dqt, model_step as MS

pytestmark = pytest.mark.gpu


def test_gradients_match_the_model_in_pytorch(lib):
    """Same weights, same batch: loss and dense gradients of the two paths.
    They differ by bf16 roundings in other places (2^-8 each, of which a
    layer has about ten), by int8 codes that fall to the other side, and by the
    gate and up checkpoints (a group's maximum / 254 at most, about 1 % of the
    gradients through them): 5 % of a gradient's norm covers two layers."""
    own = MS.DQTModel(dataclasses.replace(MS.MODELS["tiny"], own_ops=True))
    ref = MS.DQTModel(MS.MODELS["tiny"])
    tok, tgt = MS.synthetic_batch(MS.MODELS["tiny"], 0)
    log("model: own operators against PyTorch")
    a, b = own.loss(tok, tgt), ref.loss(tok, tgt)
    a.backward()
    b.backward()
    a, b = float(a.detach()), float(b.detach())
    assert abs(a - b) < 2e-3 * b
    pairs = [("emb", own.emb, ref.emb), ("head", own.head, ref.head), ("final", own.final_norm, ref.final_norm)]
    for i, (x, y) in enumerate(zip(own.norms, ref.norms)):
        pairs += [(f"norm {i}.{j}", p, q) for j, (p, q) in enumerate(zip(x, y))]
    for name, p, q in pairs:
        err = float((p.grad - q.grad).norm() / q.grad.norm())
        log(f"{name}: {err:.4f}")
        assert err < 0.05, (name, err)


def test_packed_documents_stay_apart(lib):
    """A document's logits do not depend on the other documents of the batch,
    nor on where it lies in it."""
    cfg = MS.MODELS["tiny_ops"]
    model = MS.DQTModel(cfg)
    tok, _ = MS.synthetic_batch(cfg, 1)
    tok = tok.reshape(-1)
    lens = [100, 1, 0, 155]
    starts = torch.tensor([0, 100, 101, 101, 256], dtype=torch.int32, device=DEV)
    log("model: packed documents")
    with torch.no_grad():
        a = model.logits(tok, starts)
        other = tok.clone()
        other[:100] = (other[:100] + 7) % cfg.vocab
        b = model.logits(other, starts)
        assert torch.equal(a[100:], b[100:]) and not torch.equal(a[:100], b[:100])
        docs = torch.split(tok, lens)
        turned = torch.cat([docs[3], docs[0], docs[1]])
        c = model.logits(turned, torch.tensor([0, 155, 255, 256], dtype=torch.int32, device=DEV))
        # (only the LM head's library product may sum in another order: one bf16 step)
        assert torch.allclose(c[:155].float(), a[101:].float(), rtol=2.0 ** -7, atol=2.0 ** -7 * float(a.float().abs().max()))


def test_padded_batch(lib):
    """Tokens outside every document change nothing in the documents, and with
    targets outside the vocabulary nothing in the loss or the weights."""
    cfg = MS.MODELS["tiny_ops"]
    tok, tgt = MS.synthetic_batch(cfg, 3)
    tgt.view(-1)[:16] = -100
    tgt.view(-1)[200:] = -100
    s32 = lambda *x: torch.tensor(x, dtype=torch.int32, device=DEV)
    log("model: a padded batch")
    got = []
    for starts, pad in ((s32(16, 100, 200), 5), (s32(16, 100, 200), 77), (s32(0, 16, 100, 200, 256), 5)):
        model = MS.DQTModel(cfg)
        t = tok.clone().view(-1)
        t[:16] = pad
        t[200:] = pad
        loss = model.train_step(t.view_as(tok), tgt, starts)
        codes = [c.clone() for layer in model.groups for g in layer.values() for c in g.codes]
        assert int(model.counters[1]) == 0 and bool(loss.isfinite())
        got.append((loss, codes))
    for loss, codes in got[1:]:
        assert torch.equal(loss, got[0][0])
        assert all(torch.equal(a, b) for a, b in zip(codes, got[0][1]))


def test_score_matches_log_softmax(lib):
    cfg = MS.MODELS["tiny_ops"]
    model = MS.DQTModel(cfg)
    tok, tgt = MS.synthetic_batch(cfg, 2)
    tgt[0, 5] = -100
    log("model: score")
    out = model.score(tok, tgt, top_k=7)
    with torch.no_grad():
        x = model.logits(tok).double()
    lp = torch.log_softmax(x, -1)
    want = lp.gather(1, tgt.reshape(-1, 1).clamp(min=0)).view(cfg.batch, cfg.seq)
    want[0, 5] = 0.0
    assert out["logp"].shape == (cfg.batch, cfg.seq) and out["top_ids"].shape == (cfg.batch, cfg.seq, 7)
    assert float((out["logp"].double() - want).abs().max()) < 1e-5
    assert float((out["entropy"].double() + (lp.exp() * lp).sum(-1).view_as(want)).abs().max()) < 1e-4
    val, idx = torch.sort(x, dim=-1, descending=True, stable=True)
    assert torch.equal(out["top_ids"].view(-1, 7), idx[:, :7])
    # the PyTorch model scores too
    ref = MS.DQTModel(MS.MODELS["tiny"])
    assert ref.score(tok, tgt)["logp"].isfinite().all()


def test_tiny_model_trains_on_packed_documents(lib):
    cfg = MS.MODELS["tiny_ops"]
    log(f"packed training steps {cfg}")
    model = MS.DQTModel(cfg)
    starts = torch.tensor([0, 37, 200, 201, 256], dtype=torch.int32, device=DEV)
    losses = []
    for s in range(3):
        tok, tgt = MS.synthetic_batch(cfg, s)
        tgt.view(-1)[torch.tensor([36, 199, 200, 255], device=DEV)] = -100    # no token follows a document's last
        losses.append(float(model.train_step(tok, tgt, starts)))
    assert all(math.isfinite(v) for v in losses) and abs(losses[0] - math.log(cfg.vocab)) < 0.5
    changed, nonfinite = model.counters.tolist()
    assert changed > 0 and nonfinite == 0


def test_configuration_refusals():
    with pytest.raises(ValueError):
        dataclasses.replace(MS.MODELS["tiny"], kv_heads=2)
    with pytest.raises(ValueError):
        dataclasses.replace(MS.MODELS["tiny_ops"], kv_heads=3)


def test_graph_replays_match_eager(lib):
    """Forward and backward of the three operators, captured together: every
    replay gives the eager results, with eager work between the replays (and
    calls of another size on the same buffers' workspaces)."""
    gen = torch.Generator(device=DEV).manual_seed(3)
    r = lambda *s, dt=torch.bfloat16: torch.randn(s, generator=gen, device=DEV).to(dt)
    T, H, KV, D, K, V = 300, 8, 2, 64, 1040, 70001
    st = torch.tensor([0, 120, 120, 300], dtype=torch.int32, device=DEV)
    one = torch.tensor([0, 1], dtype=torch.int32, device=DEV)
    long = torch.tensor([0, 9000], dtype=torch.int32, device=DEV)
    a = dqt.attn(T, T, H, KV, D, st, st)
    a1 = dqt.attn(1, 9000, H, KV, D, one, long)            # one token: keys split over blocks
    assert dqt.dqt_attn_fwd_workspace(a1) > 0 and dqt.dqt_logprob_workspace(4, V, 5) > 0
    q, k, v, do = r(T, H, D), r(T, KV, D), r(T, KV, D), r(T, H, D)
    q1, k1, v1 = r(1, H, D), r(9000, KV, D), r(9000, KV, D)
    G, U, dh = r(T, K), r(T, K), r(T, K)
    X, tgt = r(4, V, dt=torch.float32), torch.tensor([3, -1, 9000, 77], device=DEV)
    dl = torch.randn((4,), generator=gen, device=DEV)

    def bufs():
        f = lambda *s, dt=torch.float32: torch.zeros(s, dtype=dt, device=DEV)
        bf = torch.bfloat16
        return dict(O=f(T, H, D, dt=bf), lse=f(H, T), dQ=f(T, H, D, dt=bf), dK=f(T, KV, D, dt=bf), dV=f(T, KV, D, dt=bf),
                    O1=f(1, H, D, dt=bf), Xq=f(T, K, dt=torch.int8), xdq=f(T), dG=f(T, K, dt=bf), dU=f(T, K, dt=bf),
                    logp=f(4), stat=f(4, 2), ent=f(4), ids=f(4, 5, dt=torch.int64), tl=f(4, 5), dX=f(4, V))

    ck = dqt.swiglu_ckpt(T, K)
    ws = dqt.workspace(max(dqt.dqt_attn_bwd_workspace(a), dqt.dqt_attn_fwd_workspace(a), dqt.dqt_attn_fwd_workspace(a1),
                           dqt.dqt_logprob_workspace(4, V, 5)))

    def calls(b):
        dqt.dqt_attn_fwd(a, q, k, v, b["O"], b["lse"], ws)
        dqt.dqt_attn_bwd(a, q, k, v, b["O"], b["lse"], do, b["dQ"], b["dK"], b["dV"], ws)
        dqt.dqt_attn_fwd(a1, q1, k1, v1, b["O1"], None, ws)
        dqt.dqt_swiglu_act_quant(G, U, dqt.DQT_I8, b["Xq"], b["xdq"], ck)
        dqt.dqt_swiglu_backward_ckpt(dh, ck, b["dG"], b["dU"])
        dqt.dqt_logprob_fwd(X, tgt, b["logp"], None, b["ent"], b["stat"], b["ids"], b["tl"], ws)
        dqt.dqt_logprob_bwd(X, tgt, b["stat"], dl, b["dX"])

    eager, g = bufs(), bufs()
    calls(eager)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        calls(g)
    torch.cuda.synchronize()
    for rep in range(3):
        log(f"graph replay {rep}")
        for t in g.values():
            t.zero_()
        ws.fill_(float("nan"))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for n in g:
            assert torch.equal(g[n], eager[n]), (rep, n)


def test_calls_on_another_stream(lib):
    """Each call takes the stream it is given; results equal the default stream's."""
    gen = torch.Generator(device=DEV).manual_seed(4)
    G, U = (torch.randn((70, 512), generator=gen, device=DEV) for _ in range(2))
    X = torch.randn((70, 3001), generator=gen, device=DEV)
    t = torch.randint(0, 3001, (70,), generator=gen, device=DEV)

    def go(stream):
        o = dict(Xq=torch.zeros((70, 512), dtype=torch.uint8, device=DEV), xdq=torch.zeros((70,), device=DEV),
                 logp=torch.zeros((70,), device=DEV), stat=torch.zeros((70, 2), device=DEV), dX=torch.zeros_like(X),
                 dG=torch.zeros_like(G), dU=torch.zeros_like(G))
        ws = dqt.workspace(dqt.dqt_logprob_workspace(70, 3001))
        torch.cuda.synchronize()
        dqt.dqt_swiglu_act_quant(G, U, dqt.DQT_FP8E4M3, o["Xq"], o["xdq"], stream=stream)
        dqt.dqt_swiglu_backward(G, G, U, o["dG"], o["dU"], stream=stream)
        dqt.dqt_logprob_fwd(X, t, o["logp"], stat=o["stat"], ws=ws, stream=stream)
        dqt.dqt_logprob_bwd(X, t, o["stat"], o["logp"], o["dX"], stream=stream)
        torch.cuda.synchronize()
        return o

    log("operators on another stream")
    a, b = go(None), go(torch.cuda.Stream())
    for n in a:
        assert torch.equal(a[n], b[n]), n


def test_strided_targets(lib):
    """Targets that are every second value of a tensor: loss, gradients and
    scores of their contiguous copy."""
    cfg = MS.MODELS["tiny_ops"]
    tok, tgt = MS.synthetic_batch(cfg, 4)
    both = torch.stack((tok, tgt), dim=-1)
    log("model: strided targets")
    got = []
    for t in (tgt, both[..., 1]):
        model = MS.DQTModel(cfg)
        out = model.score(tok, t, top_k=2)
        loss = model.loss(tok, t)
        loss.backward()
        got.append([loss.detach(), *out.values(), model.head.grad])
    for x, y in zip(*got):
        # (the head's gradient: a library product, which may sum in another order, to bf16)
        assert torch.equal(x, y) if x is not got[0][-1] else (x - y).norm() <= 2.0 ** -7 * x.norm()


@pytest.mark.parametrize("ckpt8", [True, False])
def test_what_the_feed_forward_holds_for_its_backward(lib, monkeypatch, ckpt8):
    """Gradients of gate and up: of their values in bf16, or of those that the
    8-bit checkpoints hold; the forward is the same."""
    cfg = dataclasses.replace(MS.MODELS["tiny_ops"], ckpt8=ckpt8)
    model = MS.DQTModel(cfg)
    gen = torch.Generator().manual_seed(60)
    gate, up = (torch.randn((200, cfg.ffn), generator=gen).to(torch.bfloat16) for _ in range(2))
    dy = (torch.randn((200, cfg.hidden), generator=gen) * 1e-2).to(torch.bfloat16).to(DEV)
    seen = []
    plain = MS._group_bwd
    monkeypatch.setattr(MS, "_group_bwd", lambda *a: seen.append(plain(*a)) or seen[-1])
    g, u = (t.to(DEV).requires_grad_() for t in (gate, up))
    grp = model.groups[0]["mlp_hidden"]
    log(f"model: feed-forward held in 8 bits: {ckpt8}")
    with torch.no_grad():
        Xq, xdq = torch.empty((200, cfg.ffn), dtype=torch.int8, device=DEV), torch.empty((200,), device=DEV)
        dqt.dqt_swiglu_act_quant(g, u, dqt.DQT_I8, Xq, xdq)
        (want,) = MS._group_fwd(grp, Xq, xdq)
    (y,) = MS._OwnFns.get()[1].apply(g, u, grp)
    assert torch.equal(y, want)
    y.backward(dy)
    if ckpt8:
        gate, up = (R.checkpoint_values(*R.checkpoint(t)) for t in (gate, up))
    (dh,) = seen[0]
    rg, ru, tg, tu = R.swiglu_backward(dh.cpu(), gate, up)
    for got, ref, t in ((g.grad, rg, tg), (u.grad, ru, tu)):
        assert ((got.double().cpu() - ref).abs() <= R.BF16 * ref.abs() * (1 + 2.0 ** -7) + t + 1e-37).all()
