"""Train step of a LLaMA-shaped model whose block linears are DQT layers.

Sec. 4.1 trains LLaMA-structured models (RMSNorm, rotary position
embeddings, SwiGLU feed-forward) in which every weight matrix of the blocks
is a DQT layer: low-bit codes with a fixed per-tensor scale, 8-bit
activations in the forward (Sec. 3.2), and the stochastic-rounding update of
Eq. 5 applied to the codes directly, with no high-precision copy.  This
module runs that step on one GPU.

What runs where:
  * The seven linears of each block (q, k, v, o, gate, up, down) run in this
    library's kernels through its C ABI.  Linears that share an input form
    one group: its input is quantised once (the block norms and the
    quantisation are one fused launch, dqt_rmsnorm_act_quant), its forward is
    one batched call, and its backward is one call (dqt_linear_bwd_sr_batch)
    that forms dX and applies Eq. 5 to the codes in the dW product's
    epilogue, so dW never reaches memory.  A layer's codes are not read again
    in the step once its backward has run, so updating them there is the
    step's update.
  * The rest is the environment the linears are trained in, in PyTorch:
    token embedding and LM head (dense bf16 compute, fp32 master weights
    trained by AdamW, as BitNet-style models keep them), causal attention
    (PyTorch's flash kernels), the rotary embedding, SiLU, the residual adds,
    the backward of the norms and the loss.
  * With own_ops, attention, the SwiGLU product and the loss run in this
    library too: dqt_attn_fwd / _bwd take documents of different lengths packed
    into the batch and grouped key heads; dqt_swiglu_act_quant feeds the down
    projection and keeps gate and up as 8-bit checkpoints, from which
    dqt_swiglu_backward takes their gradients (2 bytes per element of a token's
    feed-forward held for the backward, 6 in PyTorch; with ckpt8 = False gate and
    up themselves, 4 bytes); dqt_logprob_fwd / _bwd give the loss and the logits'
    gradient.

Initialisation (untimed): codes by Eq. 2-4 for the ternary grid from
W0 ~ N(0, 0.02) (alpha = mean |W0|, q = Clip(Round(W0 / alpha), -1, 1));
embedding and head N(0, 0.02); norm weights 1.
"""

from __future__ import annotations

import math
from dataclasses import dataclass

from . import dqt


@dataclass(frozen=True)
class ModelConfig:
    name: str
    layers: int
    hidden: int
    heads: int
    ffn: int
    vocab: int
    batch: int
    seq: int
    lr: float
    eps: float = 1e-6
    rope_base: float = 10000.0
    seed: int = 0
    kv_heads: int = 0          # key heads (0: as many as heads); fewer need own_ops
    own_ops: bool = False      # attention, SwiGLU and loss in this library's kernels
    # own_ops: gate and up are held for the backward in 8 bits, one scale for 128
    # elements (the forward is the same; gradients through the product are off by
    # 0.7 % rms for normal values); False: as they are, in bf16
    ckpt8: bool = True

    def __post_init__(self):
        if self.kv_heads and (self.heads % self.kv_heads or (self.kv_heads != self.heads and not self.own_ops)):
            raise ValueError("kv_heads must divide heads, and grouped heads need own_ops")

    @property
    def n_kv(self) -> int:
        return self.kv_heads or self.heads

    @property
    def tokens(self) -> int:
        return self.batch * self.seq

    def linears(self):
        """(group name, [(linear name, d_in, d_out)]) of one block; linears in
        one group share their input."""
        h, f = self.hidden, self.ffn
        kv = h // self.heads * self.n_kv
        return [("attn_in", [("q", h, h), ("k", h, kv), ("v", h, kv)]),
                ("attn_out", [("o", h, h)]),
                ("mlp_in", [("gate", h, f), ("up", h, f)]),
                ("mlp_hidden", [("down", f, h)])]

    @property
    def dqt_weights(self) -> int:
        return self.layers * sum(di * do for _, g in self.linears() for _, di, do in g)

    def step_flops(self) -> dict:
        """Algorithmic flops of one train step (forward + backward)."""
        T = self.tokens
        lin = 6 * T * self.dqt_weights
        head = 6 * T * self.vocab * self.hidden
        # causal attention: Q K^T and P V over the lower triangle, backward twice the forward
        attn = 3 * 2 * self.batch * self.seq * self.seq * self.hidden * self.layers
        return {"dqt_linears": lin, "lm_head": head, "attention": attn,
                "total": lin + head + attn}


MODELS = {
    # 24 layers, hidden 2048, 16 heads, FFN 5632, vocab 32000; 8 x 2048 tokens
    "llama24_h2048": ModelConfig(name="llama24_h2048", layers=24, hidden=2048, heads=16,
                                 ffn=5632, vocab=32000, batch=8, seq=2048, lr=3e-4),
    # a small model of the same structure, for tests
    "tiny": ModelConfig(name="tiny", layers=2, hidden=256, heads=4, ffn=512, vocab=1000,
                        batch=2, seq=128, lr=3e-4),
    # the same two with attention, SwiGLU and loss in this library's kernels
    "llama24_h2048_ops": ModelConfig(name="llama24_h2048_ops", layers=24, hidden=2048, heads=16,
                                     ffn=5632, vocab=32000, batch=8, seq=2048, lr=3e-4, own_ops=True),
    "tiny_ops": ModelConfig(name="tiny_ops", layers=2, hidden=256, heads=4, kv_heads=2, ffn=512,
                            vocab=1000, batch=2, seq=128, lr=3e-4, own_ops=True),
}


# blocks of the norm backward (each one sums the gamma gradient of its rows)
MS_NORM_BLOCKS = 1024


def _pack_ternary_dev(q):
    """int8 codes {-1, 0, 1} [d_out, d_in] -> packed bytes [d_out, d_in / 4]:
    code q + 1 of weight k at bits 2 (k mod 4) of byte k / 4."""
    torch = dqt._torch()
    c = (q + 1).to(torch.uint8).view(q.shape[0], -1, 4)
    return (c[..., 0] | (c[..., 1] << 2) | (c[..., 2] << 4) | (c[..., 3] << 6)).contiguous()


class _Group:
    """The DQT linears of one block that share an input."""

    def __init__(self, model, layer: int, gname: str, lins):
        torch = dqt._torch()
        self.model = model
        self.layer = layer
        self.gname = gname
        self.d_in = lins[0][1]
        self.d_outs = [do for _, _, do in lins]
        self.weights, self.codes = [], []
        dev = model.dev
        for name, d_in, d_out in lins:
            tid = model.next_tensor_id()
            g = torch.Generator(device=dev)
            g.manual_seed(model.cfg.seed * 1_000_003 + tid)
            W0 = torch.randn((d_out, d_in), generator=g, device=dev, dtype=torch.float32) * 0.02
            alpha = float(W0.double().abs().mean())          # Eq. 2: AbsMean of W0
            q = torch.clamp(torch.round(W0 / alpha), -1, 1).to(torch.int8)   # Eq. 3-4, Q_p = 1
            del W0
            self.codes.append(_pack_ternary_dev(q))
            self.weights.append(dqt.weight(d_out, d_in, dqt.DQT_TERNARY2, -1, 1, alpha, tid))


def _group_fwd(grp, Xq, xdq):
    """The group's linears on their quantised input: bf16 outputs."""
    torch = dqt._torch()
    T = Xq.shape[0]
    Ys = [torch.empty((T, d_out), dtype=torch.bfloat16, device=Xq.device) for d_out in grp.d_outs]
    io = dqt.linear_io([dict(w=w, Wq=c, Xq=Xq, xdq=xdq, Y=Y)
                        for w, c, Y in zip(grp.weights, grp.codes, Ys)])
    dqt.dqt_linear_fwd_batch(io, T, dqt.DQT_I8, dqt.DQT_BF16,
                             grp.model.workspace(dqt.dqt_linear_fwd_batch_workspace(io)))
    return Ys


def _group_bwd(grp, Xq, xdq, dYs):
    """dX of each of the group's linears (bf16); the codes are updated by Eq. 5."""
    torch = dqt._torch()
    m = grp.model
    T = Xq.shape[0]
    dXs = [torch.empty((T, grp.d_in), dtype=torch.bfloat16, device=Xq.device) for _ in grp.d_outs]
    ents = []
    for w, c, dY, dX, d_out in zip(grp.weights, grp.codes, dYs, dXs, grp.d_outs):
        if dY is None:
            dY = torch.zeros((T, d_out), dtype=torch.bfloat16, device=Xq.device)
        ents.append(dict(w=w, Wq=c, Xq=Xq, xdq=xdq, dY=dY.contiguous(), dX=dX))
    io = dqt.linear_io(ents)
    dqt.dqt_linear_bwd_sr_batch(io, T, dqt.DQT_I8, dqt.DQT_BF16, dqt.DQT_BF16, dqt.DQT_BF16, m.cfg.lr,
                                m.cfg.seed, m.step_no, m.counters,
                                m.workspace(dqt.dqt_linear_bwd_batch_workspace(io, T)))
    return dXs


class _DQTGroupFn:
    """Autograd function of one group: x (or RMSNorm(x) * gamma) is quantised
    to int8 per token and fed to the group's linears; the backward returns
    dX (the quantiser passes the gradient through, and the norm's backward is
    taken here) and updates the codes by Eq. 5."""

    _cls = None

    @classmethod
    def get(cls):
        if cls._cls is not None:
            return cls._cls
        torch = dqt._torch()

        class Fn(torch.autograd.Function):
            @staticmethod
            def forward(ctx, x, gamma, grp):
                m = grp.model
                T = x.shape[0]
                Xq = torch.empty(x.shape, dtype=torch.int8, device=x.device)
                xdq = torch.empty((T,), dtype=torch.float32, device=x.device)
                rinv = None
                if gamma is None:
                    dqt.dqt_act_quant(x, dqt.DQT_I8, Xq, xdq)
                else:
                    rinv = torch.empty((T,), dtype=torch.float32, device=x.device)
                    dqt.dqt_rmsnorm_act_quant(x, gamma, m.cfg.eps, dqt.DQT_I8, Xq, xdq, rinv)
                Ys = _group_fwd(grp, Xq, xdq)
                ctx.grp = grp
                ctx.has_gamma = gamma is not None
                if gamma is None:
                    ctx.save_for_backward(Xq, xdq)
                else:
                    ctx.save_for_backward(Xq, xdq, x, gamma, rinv)
                return tuple(Ys)

            @staticmethod
            def backward(ctx, *dYs):
                saved = ctx.saved_tensors
                Xq, xdq = saved[0], saved[1]
                dXs = _group_bwd(ctx.grp, Xq, xdq, dYs)
                if not ctx.has_gamma:
                    if len(dXs) == 1:
                        return dXs[0], None, None
                    dn = dXs[0].float()
                    for d in dXs[1:]:
                        dn += d.float()
                    return dn.to(torch.bfloat16), None, None
                # the norm's backward (y = x r gamma, r = (mean(x^2) + eps)^(-1/2))
                # on the sum of the linears' dX, in one kernel; the gamma
                # gradient from its per-block partial sums
                x, gamma, rinv = saved[2], saved[3], saved[4]
                dx = torch.empty_like(x)
                gpart = torch.empty((MS_NORM_BLOCKS, x.shape[1]), dtype=torch.float32,
                                    device=x.device)
                dqt.dqt_rmsnorm_backward(dXs, x, gamma, rinv, dx, gpart)
                return dx, gpart.sum(0), None

        cls._cls = Fn
        return Fn


class _OwnFns:
    """Autograd functions of the operators that own_ops runs in this library."""

    _cls = None

    @classmethod
    def get(cls):
        if cls._cls is not None:
            return cls._cls
        torch = dqt._torch()

        class Attn(torch.autograd.Function):
            """softmax(q k^T / sqrt(d)) v, causal, per packed sequence; q
            [T, heads, d], k and v [T, kv heads, d]."""

            @staticmethod
            def forward(ctx, q, k, v, starts, model):
                T, nh, d = q.shape
                a = dqt.attn(T, T, nh, k.shape[1], d, starts, starts)
                o = torch.empty((T, nh, d), dtype=torch.bfloat16, device=q.device)
                lse = torch.empty((nh, T), dtype=torch.float32, device=q.device)
                dqt.dqt_attn_fwd(a, q, k, v, o, lse, model.workspace(dqt.dqt_attn_fwd_workspace(a)))
                ctx.a, ctx.model = a, model
                ctx.save_for_backward(q, k, v, o, lse)
                return o

            @staticmethod
            def backward(ctx, do):
                q, k, v, o, lse = ctx.saved_tensors
                dq = torch.empty(q.shape, dtype=torch.bfloat16, device=q.device)
                dk, dv = (torch.empty(k.shape, dtype=torch.bfloat16, device=q.device) for _ in range(2))
                dqt.dqt_attn_bwd(ctx.a, q, k, v, o, lse, do.contiguous(), dq, dk, dv,
                                 ctx.model.workspace(dqt.dqt_attn_bwd_workspace(ctx.a)))
                return dq, dk, dv, None, None

        class SwigluGroup(torch.autograd.Function):
            """silu(gate) * up, quantised and fed to the group's linears (the
            down projection); gate and up are kept as 8-bit checkpoints, or as
            they are (ckpt8 = False)."""

            @staticmethod
            def forward(ctx, gate, up, grp):
                T, K = gate.shape
                Xq = torch.empty((T, K), dtype=torch.int8, device=gate.device)
                xdq = torch.empty((T,), dtype=torch.float32, device=gate.device)
                gate, up = gate.contiguous(), up.contiguous()
                ckpt = dqt.swiglu_ckpt(T, K, gate.device) if grp.model.cfg.ckpt8 else None
                dqt.dqt_swiglu_act_quant(gate, up, dqt.DQT_I8, Xq, xdq, ckpt)
                ctx.grp = grp
                kept = (gate, up) if ckpt is None else (ckpt.Gq, ckpt.Uq, ckpt.gs, ckpt.us)
                ctx.save_for_backward(Xq, xdq, *kept)
                return tuple(_group_fwd(grp, Xq, xdq))

            @staticmethod
            def backward(ctx, *dYs):
                Xq, xdq, *kept = ctx.saved_tensors
                dXs = _group_bwd(ctx.grp, Xq, xdq, dYs)
                dh = dXs[0]
                for d in dXs[1:]:
                    dh = dh + d
                dg, du = torch.empty_like(dh), torch.empty_like(dh)
                if len(kept) == 2:
                    dqt.dqt_swiglu_backward(dh, *kept, dg, du)
                else:
                    dqt.dqt_swiglu_backward_ckpt(dh, dqt.SwigluCkpt(*kept), dg, du)
                return dg, du, None

        class TokenLoss(torch.autograd.Function):
            """Mean of -log p(target) over the rows that have a target (one in
            0 .. V - 1)."""

            @staticmethod
            def forward(ctx, logits, targets, model):
                M, V = logits.shape
                logp = torch.empty((M,), dtype=torch.float32, device=logits.device)
                stat = torch.empty((M, 2), dtype=torch.float32, device=logits.device)
                dqt.dqt_logprob_fwd(logits, targets, logp, stat=stat,
                                    ws=model.workspace(dqt.dqt_logprob_workspace(M, V)))
                n = ((targets >= 0) & (targets < V)).sum().clamp(min=1).float()
                ctx.save_for_backward(logits, targets, stat, n)
                return -logp.sum() / n

            @staticmethod
            def backward(ctx, dloss):
                logits, targets, stat, n = ctx.saved_tensors
                dlogp = (-dloss.float() / n).expand(logits.shape[0]).contiguous()
                dx = torch.empty_like(logits)
                dqt.dqt_logprob_bwd(logits, targets, stat, dlogp, dx)
                return dx, None, None

        cls._cls = (Attn, SwigluGroup, TokenLoss)
        return cls._cls


class DQTModel:
    """Parameters and train step of a LLaMA-shaped model with DQT linears."""

    def __init__(self, cfg: ModelConfig, device="cuda:0"):
        torch = dqt._torch()
        dqt.load()
        self.cfg = cfg
        self.dev = device
        self._tid = 0
        self.step_no = 0
        self._ws = None
        self.counters = torch.zeros((2,), dtype=torch.int64, device=device)
        g = torch.Generator(device=device)
        g.manual_seed(cfg.seed)
        H, V = cfg.hidden, cfg.vocab
        P = torch.nn.Parameter
        self.emb = P(torch.randn((V, H), generator=g, device=device) * 0.02)
        self.head = P(torch.randn((V, H), generator=g, device=device) * 0.02)
        self.final_norm = P(torch.ones((H,), device=device))
        self.norms = []
        self.groups = []
        for layer in range(cfg.layers):
            self.norms.append((P(torch.ones((H,), device=device)), P(torch.ones((H,), device=device))))
            self.groups.append({gname: _Group(self, layer, gname, lins)
                                for gname, lins in cfg.linears()})
        dense = [self.emb, self.head, self.final_norm] + [p for n in self.norms for p in n]
        self.opt = torch.optim.AdamW(dense, lr=cfg.lr, betas=(0.9, 0.95), weight_decay=0.1)
        hd = H // cfg.heads
        inv = 1.0 / (cfg.rope_base ** (torch.arange(0, hd, 2, device=device, dtype=torch.float32) / hd))
        # (packed documents may be as long as the batch)
        rows = cfg.tokens if cfg.own_ops else cfg.seq
        ang = torch.arange(rows, device=device, dtype=torch.float32)[:, None] * inv[None, :]
        self.cos = torch.cos(ang).to(torch.bfloat16)[None, None]   # [1, 1, rows, hd/2]
        self.sin = torch.sin(ang).to(torch.bfloat16)[None, None]
        # first token of each of the batch's sequences, and behind the last
        self.starts = torch.arange(0, cfg.tokens + 1, cfg.seq, dtype=torch.int32, device=device)

    def next_tensor_id(self) -> int:
        t = self._tid
        self._tid += 1
        return t

    def workspace(self, nbytes: int):
        """One device workspace for every call (calls on one stream run in
        order); grown when a call needs more."""
        if nbytes == 0:
            return None
        if self._ws is None or self._ws.numel() * 4 < nbytes:
            self._ws = dqt.workspace(nbytes, self.dev)
        return self._ws

    def _rope(self, x, c=None, s=None):
        # x [B, nh, S, hd] (or [T, nh, hd] with each token's c and s): rotate
        # the two halves of each head
        h = x.shape[-1] // 2
        x1, x2 = x[..., :h], x[..., h:]
        if c is None:
            c, s = self.cos, self.sin
        return self._cat((x1 * c - x2 * s, x1 * s + x2 * c))

    @staticmethod
    def _cat(parts):
        return dqt._torch().cat(parts, dim=-1)

    def logits(self, tokens, starts=None):
        """Logits [tokens, vocab] (bf16) of one batch.  starts (own_ops): int32
        on the device, the first token of each document packed into the batch and,
        last, the token behind the last document; by default the batch's sequences.
        Tokens behind it (or before the first document) pad the batch: they see
        each other alone, and take no part in a loss whose targets there are
        outside the vocabulary."""
        torch = dqt._torch()
        F = torch.nn.functional
        from torch.nn.attention import SDPBackend, sdpa_kernel
        cfg = self.cfg
        B, S, H, nh = cfg.batch, cfg.seq, cfg.hidden, cfg.heads
        hd = H // nh
        fn = _DQTGroupFn.get()
        if cfg.own_ops:
            attn_fn, swiglu_fn, _ = _OwnFns.get()
            if starts is None:
                starts = self.starts
            else:      # (padding forms sequences of its own, mostly empty: every row is written)
                starts = torch.cat((self.starts[:1], starts, self.starts[-1:]))
            tok = torch.arange(B * S, dtype=torch.int32, device=self.dev)
            pos = (tok - starts[torch.searchsorted(starts[1:], tok, right=True)]).long()
            cos, sin = self.cos[0, 0, pos][:, None], self.sin[0, 0, pos][:, None]
        elif starts is not None:
            raise ValueError("packed documents need own_ops")
        h = F.embedding(tokens.reshape(-1), self.emb.to(torch.bfloat16))     # [T, H] bf16
        for layer in range(cfg.layers):
            grp = self.groups[layer]
            n_attn, n_mlp = self.norms[layer]
            q, k, v = fn.apply(h, n_attn, grp["attn_in"])
            if cfg.own_ops:
                q, k, v = (t.view(B * S, -1, hd) for t in (q, k, v))
                a = attn_fn.apply(self._rope(q, cos, sin), self._rope(k, cos, sin), v, starts, self)
                a = a.view(B * S, H)
            else:
                q, k, v = (t.view(B, S, nh, hd).transpose(1, 2) for t in (q, k, v))
                q, k = self._rope(q), self._rope(k)
                # flash / memory-efficient kernels only (no fallback to the math path)
                with sdpa_kernel([SDPBackend.FLASH_ATTENTION, SDPBackend.EFFICIENT_ATTENTION]):
                    a = F.scaled_dot_product_attention(q, k, v, is_causal=True)
                a = a.transpose(1, 2).reshape(B * S, H)
            (o,) = fn.apply(a, None, grp["attn_out"])
            h = h + o
            gt, up = fn.apply(h, n_mlp, grp["mlp_in"])
            if cfg.own_ops:
                (d,) = swiglu_fn.apply(gt, up, grp["mlp_hidden"])
            else:
                (d,) = fn.apply(F.silu(gt) * up, None, grp["mlp_hidden"])
            h = h + d
        hn = F.rms_norm(h.float(), (H,), weight=self.final_norm, eps=cfg.eps).to(torch.bfloat16)
        return hn @ self.head.to(torch.bfloat16).t()

    def loss(self, tokens, targets, starts=None):
        """Forward of one batch: mean next-token cross-entropy (fp32).  targets:
        int64 on the device, one a token, of any strides.  With own_ops every
        target outside the vocabulary is padding (the PyTorch form takes -100 alone
        and refuses others), and a batch of nothing else has loss 0 (there NaN)."""
        logits = self.logits(tokens, starts)
        if self.cfg.own_ops:
            return _OwnFns.get()[2].apply(logits, targets.reshape(-1).contiguous(), self)
        return dqt._torch().nn.functional.cross_entropy(logits.float(), targets.reshape(-1))

    def score(self, tokens, targets, top_k=0, starts=None):
        """Log probability of each target token (0 where it is outside the
        vocabulary), the entropy of each prediction and, with top_k, the ids and
        log probabilities of its most probable tokens, each [batch, seq(, top_k)].
        A continuation's score is the sum of its tokens' log probabilities,
        perplexity exp of their negated mean."""
        torch = dqt._torch()
        with torch.no_grad():
            x = self.logits(tokens, starts)
            M, V = x.shape
            f = lambda *shape: torch.empty(shape, dtype=torch.float32, device=x.device)
            out = dict(logp=f(M), entropy=f(M))
            if top_k:
                out.update(top_ids=torch.empty((M, top_k), dtype=torch.int64, device=x.device), top_logp=f(M, top_k))
            dqt.dqt_logprob_fwd(x, targets.reshape(-1).contiguous(), out["logp"], None, out["entropy"], None, out.get("top_ids"),
                                out.get("top_logp"), self.workspace(dqt.dqt_logprob_workspace(M, V, top_k)))
        return {k: v.view(self.cfg.batch, self.cfg.seq, *v.shape[1:]) for k, v in out.items()}

    def train_step(self, tokens, targets, starts=None):
        """One step: forward, backward (the DQT codes are updated by Eq. 5
        inside it, keyed by this step's number), AdamW on the dense
        parameters.  Returns the loss tensor (not synchronised)."""
        self.step_no += 1
        self.opt.zero_grad(set_to_none=True)
        loss = self.loss(tokens, targets, starts)
        loss.backward()
        self.opt.step()
        return loss.detach()


def synthetic_batch(cfg: ModelConfig, step: int, device="cuda:0"):
    """Uniform-random token ids [batch, seq] and the next-token targets."""
    torch = dqt._torch()
    g = torch.Generator(device=device)
    g.manual_seed(cfg.seed * 7919 + step)
    ids = torch.randint(0, cfg.vocab, (cfg.batch, cfg.seq + 1), generator=g, device=device)
    return ids[:, :-1].contiguous(), ids[:, 1:].contiguous()


def initial_loss_expected(cfg: ModelConfig) -> float:
    """Uniform targets: the loss of a near-uniform predictor is ln(vocab)."""
    return math.log(cfg.vocab)
