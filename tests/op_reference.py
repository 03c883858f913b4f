"""Plain float64 implementations of the model operators (attention, SwiGLU
with 8-bit checkpoints, token log probabilities), written from their formulas,
with bounds of what rounding may add.  A rounding to a type is off by at most
half a step: 2^-8 of the value for bf16, 2^-24 for fp32, 2^-4 for e4m3."""
import numpy as np
import torch

BF16, F32 = 2.0 ** -8, 2.0 ** -24


def attention(Q, K, V, q_start, k_start, scale, causal, dO=None):
    """Q [tq, heads, d], K and V [tk, kv_heads, d] (float64, CPU).  Returns a
    dict of O, lse and (with dO) dQ, dK, dV, and a bound t_* for each:

    O: p is rounded to bf16 before the second product (BF16 sum p |v|) and O
    at the end (BF16 |O|).  SLACK covers p's fp32 error: its exponent is a sum
    of d products, each rounded, and lse (d + 8 fp32 roundings of sum |q k|
    scale, about 1e-4 at the sizes here).
    dV: the same with dO for v.
    dQ, dK: g = p (dO.v - delta) is rounded to bf16; delta = dO.O is formed
    from the rounded O, so it is off by at most sum |dO| t_O."""
    SLACK = 2.0 ** -12
    Q, K, V = Q.double(), K.double(), V.double()
    tq, heads, d = Q.shape
    tk, kvh, _ = K.shape
    G = heads // kvh
    z64 = dict(dtype=torch.float64)
    r = dict(O=torch.zeros((tq, heads, d), **z64), lse=torch.full((heads, tq), -np.inf, **z64),
             t_O=torch.zeros((tq, heads, d), **z64), t_lse=torch.zeros((heads, tq), **z64))
    if dO is not None:
        dO = dO.double()
        for n, ref in (("dQ", Q), ("dK", K), ("dV", V)):
            r[n], r["t_" + n] = torch.zeros_like(ref), torch.zeros_like(ref)
    for s in range(len(q_start) - 1):
        a, b, e, f = q_start[s], q_start[s + 1], k_start[s], k_start[s + 1]
        lq, lk = b - a, f - e
        if lq == 0 or lk == 0:
            continue
        see = torch.ones((lq, lk), dtype=torch.bool)
        if causal:
            see = torch.arange(lk)[None, :] <= torch.arange(lq)[:, None] + lk - lq
        some = see.any(1)
        for h in range(heads):
            g = h // G
            q, k, v = Q[a:b, h], K[e:f, g], V[e:f, g]
            z = (scale * (q @ k.T)).masked_fill(~see, -np.inf)
            m = z.amax(1, keepdim=True)
            m[~some] = 0.0
            w = torch.exp(z - m)
            tot = w.sum(1, keepdim=True)
            p = torch.where(some[:, None], w / tot, torch.zeros_like(w))
            o = p @ v
            pv = p @ v.abs()
            t_o = BF16 * o.abs() + (BF16 + SLACK) * pv
            r["O"][a:b, h], r["t_O"][a:b, h] = o, t_o
            r["lse"][h, a:b] = torch.where(some, (m + torch.log(tot)).squeeze(1), torch.full((lq,), -np.inf, **z64))
            zz = (scale * (q.abs() @ k.abs().T)).amax(1)
            r["t_lse"][h, a:b] = (d + 16) * F32 * (zz + 1) + 8 * F32 * (lk + 1) ** 0.5
            if dO is None:
                continue
            do = dO[a:b, h]
            dp = do @ v.T
            delta = (do * o).sum(1, keepdim=True)
            ds = p * (dp - delta)
            t_ds = (BF16 + 2 * SLACK) * ds.abs() + p * (do.abs() * t_o).sum(1, keepdim=True) * (1 + BF16)
            r["dQ"][a:b, h] = scale * (ds @ k)
            r["t_dQ"][a:b, h] = scale * (t_ds @ k.abs())
            r["dK"][e:f, g] += scale * (ds.T @ q)
            r["t_dK"][e:f, g] += scale * (t_ds.T @ q.abs())
            r["dV"][e:f, g] += p.T @ do
            r["t_dV"][e:f, g] += (BF16 + SLACK) * (p.T @ do.abs())
    if dO is not None:
        for n in ("dQ", "dK", "dV"):
            r["t_" + n] += BF16 * r[n].abs() * (1 + BF16)
    return r


def swiglu(G, U):
    """h in float64.  In fp32 (exp within 2 units in the last place, then an
    addition, a division and a product) it is off by at most 8 F32 |h|."""
    G, U = G.double(), U.double()
    return G / (1 + torch.exp(-G)) * U


H_REL = 8 * F32


def checkpoint(x):
    """fp32 arithmetic, one rounding per operation: (codes, scales)."""
    x = x.float().numpy()
    M, K = x.shape
    n = (K + 127) // 128
    codes, scales = np.zeros((M, K), np.int8), np.zeros((M, n), np.float32)
    for g in range(n):
        y = x[:, 128 * g:128 * g + 128]
        a = np.maximum(np.abs(y).max(1), np.float32(1e-5)).astype(np.float32)
        inv = np.float32(127) / a
        codes[:, 128 * g:128 * g + 128] = np.clip(np.rint(y * inv[:, None]), -128, 127)
        scales[:, g] = a / np.float32(127)
    return codes, scales


def checkpoint_values(codes, scales):
    """code times scale, in fp32 as the backward forms it, then float64."""
    s = np.repeat(scales, 128, axis=1)[:, :codes.shape[1]]
    return torch.from_numpy((codes.astype(np.float32) * s).astype(np.float64))


def swiglu_backward(dH, g, u):
    """float64 dG, dU and what fp32 arithmetic adds: 1 - s and 1 + g (1 - s)
    may cancel, each to 4 F32 of its terms, on top of 8 roundings."""
    dH, g, u = dH.double(), g.double(), u.double()
    s = 1 / (1 + torch.exp(-g))
    dU = dH * g * s
    dG = dH * u * s * (1 + g * (1 - s))
    return dG, dU, 16 * F32 * (dH * u).abs() * s * (1 + g.abs()), 16 * F32 * dU.abs()


def logprob(X, targets, threads=256):
    """Rows of X [M, V] (fp32 values): dict of float64 results and the relative
    error that fp32 sums and exponentials may have: V / threads terms one after
    another, 16 joins, and an exponent below 2^7 rounded twice."""
    x = X.double()
    M, V = x.shape
    m = x.amax(1, keepdim=True)
    none = torch.isinf(m) & (m < 0)
    m = torch.where(none, torch.zeros_like(m), m)
    e = torch.exp(x - m)
    s = e.sum(1, keepdim=True)
    d = (x - m) - torch.log(s)         # (not x - lse, which large logits would cancel)
    lse = (m + torch.log(s)).squeeze(1)
    p = torch.where(none, torch.zeros_like(e), e / s)
    plogp = torch.where(p > 0, p * d, torch.zeros_like(p))
    has = (targets >= 0) & (targets < V)
    dt = d.gather(1, targets.clamp(0, V - 1)[:, None]).squeeze(1)
    logp = torch.where(has, torch.where(none.squeeze(1), torch.full_like(lse, -np.inf), dt), torch.zeros_like(lse))
    rel = (V / threads + 16 + 128) * F32
    # log s, below 2^6: its own rounding; lse: the sum's too
    t_d = rel + 2.0 ** 7 * F32
    t_lse = t_d + F32 * torch.where(none.squeeze(1), torch.zeros_like(lse), lse.abs())
    return dict(lse=lse, logp=logp, entropy=-plogp.sum(1), p=p, plogp=plogp, d=d, has=has, t_lse=t_lse, t_d=t_d,
                t_logp=t_d + 2 * F32 * torch.where(has & torch.isfinite(dt), dt.abs(), torch.zeros_like(lse)),
                t_entropy=4 * rel * (2 + (-plogp.sum(1)).abs()) + 4 * F32 * V ** 0.5)
