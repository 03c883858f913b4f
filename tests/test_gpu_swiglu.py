"""SwiGLU fused with the 8-bit quantisation, its 8-bit checkpoints and its
backward, against plain float64 / fp32 arithmetic."""
import numpy as np
import pytest
import torch

import op_reference as R
from gpu_util import DEV, log
from paper_2412_04787_amd import dqt

pytestmark = pytest.mark.gpu

SIZES = [(1, 16), (3, 48), (5, 128), (9, 144), (130, 2048), (7, 2064), (33, 4096), (4, 5632), (3, 8192), (2, 11008),
         (2, 16384), (2, 16400)]


def inputs(M, K, dt, seed):
    g = torch.Generator().manual_seed(seed)
    G, U = (torch.randn((M, K), generator=g) for _ in range(2))
    G *= torch.exp(torch.linspace(-3, 3, M))[:, None]       # magnitudes across rows
    if M > 2:
        U[M // 2] = 0.0                                     # a zero row
        G[1, :8] = torch.tensor([-100.0, 100.0, -88.5, 0.0, -0.0, 30.0, -30.0, 1e-30])
    dH = torch.randn((M, K), generator=g) * 1e-2
    return [t.to(dt) for t in (G, U, dH)]


@pytest.mark.parametrize("dt", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("act", ["i8", "e4m3"])
@pytest.mark.parametrize("M,K", SIZES)
def test_swiglu_act_quant(lib, dt, act, M, K):
    log(f"swiglu M={M} K={K} {dt} {act}")
    G, U, _ = inputs(M, K, dt, K + M)
    code = dqt.DQT_I8 if act == "i8" else dqt.DQT_FP8E4M3
    outs = []
    for ck in (None, dqt.swiglu_ckpt(M, K)):
        Xq = torch.full((M, K), 77, dtype=torch.int8 if act == "i8" else torch.uint8, device=DEV)
        xdq = torch.empty((M,), dtype=torch.float32, device=DEV)
        dqt.dqt_swiglu_act_quant(G.to(DEV), U.to(DEV), code, Xq, xdq, ck)
        torch.cuda.synchronize()
        outs.append((Xq, xdq))
    assert torch.equal(outs[0][0], outs[1][0]) and torch.equal(outs[0][1], outs[1][1])
    h = R.swiglu(G, U)
    top = 127.0 if act == "i8" else 448.0
    m = h.abs().amax(1).clamp(min=float(np.float32(1e-5)))
    d = outs[0][1].double().cpu()
    assert ((d - m / top).abs() <= (R.H_REL + 2 * R.F32) * m / top).all()
    y = h * (top / m)[:, None]
    err = (2 * R.H_REL + 4 * R.F32) * top
    if act == "i8":
        got = outs[0][0].cpu().double()
        assert ((got - y).abs() <= 0.5 + err).all(), float((got - y).abs().max())
    else:
        got = outs[0][0].cpu().view(torch.float8_e4m3fn).double()
        assert ((got - y).abs() <= 2.0 ** -4 * y.abs() + 2.0 ** -10 + err * 2.0 ** -3).all()
    for x, q, s in ((G, ck.Gq, ck.gs), (U, ck.Uq, ck.us)):
        codes, scales = R.checkpoint(x)
        assert np.array_equal(q.cpu().numpy(), codes)
        assert np.array_equal(s.cpu().numpy(), scales)


@pytest.mark.parametrize("dt", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("stored", [True, False])
@pytest.mark.parametrize("M,K", SIZES)
def test_swiglu_backward(lib, dt, stored, M, K):
    log(f"swiglu backward M={M} K={K} {dt} checkpoint={stored}")
    G, U, dH = inputs(M, K, dt, K + M + 1)
    dG, dU = (torch.empty((M, K), dtype=dt, device=DEV) for _ in range(2))
    if stored:
        ck = dqt.swiglu_ckpt(M, K)
        (a, b), (c, e) = R.checkpoint(G), R.checkpoint(U)
        for t, v in ((ck.Gq, a), (ck.gs, b), (ck.Uq, c), (ck.us, e)):
            t.copy_(torch.from_numpy(v))
        g, u = R.checkpoint_values(a, b), R.checkpoint_values(c, e)
        dqt.dqt_swiglu_backward_ckpt(dH.to(DEV), ck, dG, dU)
    else:
        g, u = G, U
        dqt.dqt_swiglu_backward(dH.to(DEV), G.to(DEV), U.to(DEV), dG, dU)
    torch.cuda.synchronize()
    rg, ru, tg, tu = R.swiglu_backward(dH, g, u)
    half = R.BF16 if dt == torch.bfloat16 else R.F32
    for n, got, ref, t in (("dG", dG, rg, tg), ("dU", dU, ru, tu)):
        err = (got.double().cpu() - ref).abs()
        tol = half * ref.abs() * (1 + 2.0 ** -7) + t + 1e-37
        assert (err <= tol).all(), (n, float(err.max()), int((err > tol).sum()))


def test_swiglu_gradient_against_differences(lib):
    M, K = 4, 96
    G, U, dH = inputs(M, K, torch.float32, 3)
    G[1, :8] = torch.linspace(-3, 3, 8)
    dG, dU = (torch.empty((M, K), dtype=torch.float32, device=DEV) for _ in range(2))
    log("swiglu: differences")
    dqt.dqt_swiglu_backward(dH.to(DEV), G.to(DEV), U.to(DEV), dG, dU)
    torch.cuda.synchronize()
    h = 1e-5
    for got, at in ((dG, 0), (dU, 1)):
        x = [G.double(), U.double()]
        up, down = list(x), list(x)
        up[at], down[at] = x[at] + h, x[at] - h
        diff = dH.double() * (R.swiglu(*up) - R.swiglu(*down)) / (2 * h)
        # (central differences: h^2 / 6 times a third derivative below 4 |u|, and rounding 1e-16 / h |h|)
        tol = 1e-5 * diff.abs() + dH.double().abs() * 1e-8 * (1 + G.double().abs()) * (1 + U.double().abs())
        assert ((got.double().cpu() - diff).abs() <= tol).all()


def test_swiglu_backward_in_place_and_empty(lib):
    G, U, dH = inputs(5, 256, torch.bfloat16, 9)
    a, b = torch.empty((5, 256), dtype=torch.bfloat16, device=DEV), torch.empty((5, 256), dtype=torch.bfloat16, device=DEV)
    log("swiglu backward in place")
    dqt.dqt_swiglu_backward(dH.to(DEV), G.to(DEV), U.to(DEV), a, b)
    x = dH.to(DEV)
    y = torch.empty_like(x)
    dqt.dqt_swiglu_backward(x, G.to(DEV), U.to(DEV), y, x)
    torch.cuda.synchronize()
    assert torch.equal(a, y) and torch.equal(b, x)
    e = torch.empty((0, 256), dtype=torch.bfloat16, device=DEV)
    dqt.dqt_swiglu_act_quant(e, e, dqt.DQT_I8, e.to(torch.int8), torch.empty((0,), device=DEV))
    dqt.dqt_swiglu_backward(e, e, e, e, e)


@pytest.mark.parametrize("act", ["i8", "e4m3"])
def test_swiglu_codes_are_those_of_single_operations(lib, act):
    """Every finite bf16 gate, bit for bit against the same fp32 operations one
    by one; -0, gates whose exponential is huge, and tiny rows among them."""
    g = torch.arange(65536, dtype=torch.int32).to(torch.int16).view(torch.bfloat16)
    g[~torch.isfinite(g) | (g.float().abs() > 1e4)] = 0.0
    gen = torch.Generator().manual_seed(21)
    G = torch.cat([g.view(256, 256), g[torch.randperm(65536, generator=gen)].view(256, 256)])
    U = torch.randn(G.shape, generator=gen).to(torch.bfloat16)
    U[::7] *= 1e-6
    G, U = G.to(DEV), U.to(DEV)
    M, K = G.shape
    log(f"swiglu: every bf16 gate, {act}")
    Xq = torch.empty((M, K), dtype=torch.int8 if act == "i8" else torch.uint8, device=DEV)
    xdq = torch.empty((M,), dtype=torch.float32, device=DEV)
    ck = dqt.swiglu_ckpt(M, K)
    dqt.dqt_swiglu_act_quant(G, U, dqt.DQT_I8 if act == "i8" else dqt.DQT_FP8E4M3, Xq, xdq, ck)
    gf, uf = G.float(), U.float()
    h = (gf / (1.0 + torch.exp(-gf))) * uf
    top = torch.tensor(127.0 if act == "i8" else 448.0, device=DEV)
    m = h.abs().amax(1).clamp(min=float(np.float32(1e-5)))
    y = h * (top / m)[:, None]
    want = (torch.round(y).clamp(-128, 127).to(torch.int8) if act == "i8"
            else y.clamp(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8))
    torch.cuda.synchronize()
    assert torch.equal(xdq, m / top)
    assert torch.equal(Xq, want)
    for x, q, s in ((G, ck.Gq, ck.gs), (U, ck.Uq, ck.us)):
        codes, scales = R.checkpoint(x.cpu())
        assert np.array_equal(q.cpu().numpy(), codes) and np.array_equal(s.cpu().numpy(), scales)


def test_swiglu_more_rows_than_blocks(lib):
    """Rows past the largest grid give what the same rows give on their own."""
    M, K = 70001, 32
    G, U, _ = inputs(M, K, torch.bfloat16, 7)
    G, U = G.to(DEV), U.to(DEV)
    log("swiglu: 70001 rows")

    def go(g, u):
        m = g.shape[0]
        Xq, xdq = torch.empty((m, K), dtype=torch.int8, device=DEV), torch.empty((m,), dtype=torch.float32, device=DEV)
        ck = dqt.swiglu_ckpt(m, K)
        dqt.dqt_swiglu_act_quant(g, u, dqt.DQT_I8, Xq, xdq, ck)
        torch.cuda.synchronize()
        return [Xq, xdq, ck.Gq, ck.Uq, ck.gs, ck.us]

    for x, y in zip(go(G, U), go(G[65000:].contiguous(), U[65000:].contiguous())):
        assert torch.equal(x[65000:], y)


def test_swiglu_matches_unfused_quantiser(lib):
    """On rows whose product is exact in bf16, the fused call gives the codes of
    dqt_act_quant (g large: silu(g) = g in fp32)."""
    M, K = 6, 512
    gen = torch.Generator().manual_seed(1)
    G = torch.randint(32, 64, (M, K), generator=gen).to(torch.bfloat16).to(DEV)
    U = torch.tensor([-2.0, -1.0, 0.5, 0.25])[torch.randint(0, 4, (M, K), generator=gen)].to(torch.bfloat16).to(DEV)
    H = G * U
    log("swiglu: fused against the quantiser alone")
    for act, t in ((dqt.DQT_I8, torch.int8), (dqt.DQT_FP8E4M3, torch.uint8)):
        q = [torch.empty((M, K), dtype=t, device=DEV) for _ in range(2)]
        s = [torch.empty((M,), dtype=torch.float32, device=DEV) for _ in range(2)]
        dqt.dqt_swiglu_act_quant(G, U, act, q[0], s[0])
        dqt.dqt_act_quant(H, act, q[1], s[1])
        torch.cuda.synchronize()
        assert torch.equal(q[0], q[1]) and torch.equal(s[0], s[1])


def scales_of(G, U):
    """xdq of rows of which only the first gate counts, and the rows' checkpoint."""
    M, K = G.shape
    Xq, xdq = torch.empty((M, K), dtype=torch.int8, device=DEV), torch.empty((M,), dtype=torch.float32, device=DEV)
    ck = dqt.swiglu_ckpt(M, K)
    dqt.dqt_swiglu_act_quant(G, U, dqt.DQT_I8, Xq, xdq, ck)
    return xdq, ck


def test_swiglu_division_of_every_gate(lib):
    """g / (1 + exp(-g)) of every finite fp32 g >= -69 (and below it, where the
    division is another, to -104), as the row scale shows it: fl(max(|s u|, 1e-5) /
    127) with u a power of two.  The quotients are formed in 64 bits and rounded
    once, which is the correctly rounded fp32 division."""
    N, K = 1 << 23, 16
    log("swiglu: division of every gate")
    G = torch.zeros((N, K), dtype=torch.float32, device=DEV)
    U = torch.zeros((N, K), dtype=torch.float32, device=DEV)
    least = torch.tensor(1e-5, dtype=torch.float32, device=DEV)
    low = torch.arange(N, dtype=torch.int32, device=DEV)
    for sign in (0, 1):
        # 2^23 patterns a time: one exponent, every significand
        for e in range(255 if sign == 0 else 134):
            bits = low | (e << 23) | (-(1 << 31) if sign else 0)
            g = bits.view(torch.float32)
            if sign:
                g = g.clamp(min=-104.0)
            # (u keeps s u within fp32 and, but for the smallest 40 gates, above 1e-5)
            u = 2.0 ** (127 if e == 0 else 120 if e < 127 else 104 if e < 140 else 0)
            G[:, 0], U[:, 0] = g, u
            got, _ = scales_of(G, U)
            b = 1.0 + torch.exp(-g)
            s = (g.double() / b.double()).float()
            want = (torch.maximum((s * u).abs(), least).double() / 127.0).float()
            bad = got != want
            assert not bool(bad.any()), (sign, e, g[bad][:4], got[bad][:4], want[bad][:4])
            if e % 32 == 0:
                log(f"sign {sign}, exponent {e}")


def test_swiglu_checkpoint_divisions(lib):
    """fl(127 / a) and fl(a / 127) of a group's maximum a: every significand, and
    exponents from 1e-5 to the largest.  The second is the scale itself; the first
    shows in the codes of 127 values next to the borders between two codes, of
    which a step of the reciprocal's last place moves about half."""
    log("swiglu: divisions of the checkpoint")
    K, N = 128, 1 << 18
    k = torch.arange(127, dtype=torch.float64, device=DEV)[None, :] + 0.5
    gen = torch.Generator().manual_seed(50)

    def check(a):                          # a: fp32, in host memory
        inv = torch.from_numpy(np.float32(127) / a.numpy()).to(DEV)
        a = a.to(DEV)
        x = (k / inv.double()[:, None]).float()
        x = torch.minimum(x, a[:, None])
        G = torch.cat([a[:, None], x], 1)
        _, ck = scales_of(G, G)
        want = torch.round(G * inv[:, None]).clamp(-128, 127).to(torch.int8)
        assert torch.equal(ck.Gq, want) and torch.equal(ck.Uq, want)
        s = torch.from_numpy(a.cpu().numpy() / np.float32(127)).to(DEV)
        assert torch.equal(ck.gs[:, 0], s) and torch.equal(ck.us[:, 0], s)
        # (the test sees a reciprocal that is off by its last place)
        for off in (torch.nextafter(inv, inv * 2), torch.nextafter(inv, inv * 0)):
            some = (torch.round(G * off[:, None]).clamp(-128, 127).to(torch.int8) != want).any(1)
            assert some.double().mean() > 0.999

    for i in range(0, 1 << 23, N):
        check((torch.arange(i, i + N, dtype=torch.int32) | (127 << 23)).view(torch.float32))
        if i % (N * 8) == 0:
            log(f"significands from {i}")
    e = torch.randint(111, 254, (N,), generator=gen, dtype=torch.int32)
    m = torch.randint(0, 1 << 23, (N,), generator=gen, dtype=torch.int32)
    check(((e << 23) | m).view(torch.float32))
