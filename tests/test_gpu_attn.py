"""Attention over packed sequences (dqt_attn_fwd, dqt_attn_bwd) against a plain
float64 implementation: head layouts, lengths from zero to thousands, rows that
see nothing, strides, tokens outside every sequence; the gradients also against
differences."""
import numpy as np
import pytest
import torch

import op_reference as R
from gpu_util import DEV, log
from paper_2412_04787_amd import dqt

pytestmark = pytest.mark.gpu

SENT = 1.25e4          # what outputs hold before a call


def starts(lens, first=0):
    return np.concatenate([[0], np.cumsum(lens)]).astype(np.int64) + first


def tensors(gen, tokens, heads, d, layout, std=1.0):
    """A [tokens, heads, d] bf16 view: contiguous, head-major, or a slice of a
    wider buffer."""
    x = (torch.randn((tokens, heads, d), generator=gen) * std).to(torch.bfloat16)
    if layout == "heads":
        buf = x.permute(1, 0, 2).contiguous().to(DEV)
        return x, buf.permute(1, 0, 2)
    if layout == "wide":
        buf = torch.full((tokens, 3, heads + 1, d + 8), 7.0, dtype=torch.bfloat16)
        buf[:, 1, :heads, :d] = x
        return x, buf.to(DEV)[:, 1, :heads, :d]
    return x, x.to(DEV)


def like(view):
    """An output with a view's strides, filled with SENT."""
    n = 1 + sum((s - 1) * st for s, st in zip(view.shape, view.stride()))
    return torch.full((n,), SENT, dtype=torch.bfloat16, device=DEV).as_strided(view.shape, view.stride())


def close(name, got, ref, tol):
    got = got.detach().double().cpu()
    bad = ~((got - ref).abs() <= tol + 1e-30)
    bad &= ~((got == ref) & torch.isinf(ref))
    assert not bad.any(), (name, int(bad.sum()), tuple(bad.nonzero()[0].tolist()), float((got - ref).abs().max()))


def run(d, heads, kvh, lq, lk, causal=True, layout="plain", scale=None, train=True, seed=0, before=0, behind=0, std=1.0):
    gen = torch.Generator().manual_seed(seed)
    qs, ks = starts(lq, before), starts(lk, before)
    tq, tk = int(qs[-1]) + behind, int(ks[-1]) + behind
    Q, Qd = tensors(gen, tq, heads, d, layout, std)
    K, Kd = tensors(gen, tk, kvh, d, layout)
    V, Vd = tensors(gen, tk, kvh, d, layout)
    dO, dOd = tensors(gen, tq, heads, d, layout, 1e-2)
    dev32 = lambda s: torch.from_numpy(s.astype(np.int32)).to(DEV)
    a = dqt.attn(tq, tk, heads, kvh, d, dev32(qs), dev32(ks), scale=scale, causal=causal)
    O, lse = like(Qd), torch.full((heads, tq), SENT, dtype=torch.float32, device=DEV)
    ws = dqt.workspace(dqt.dqt_attn_fwd_workspace(a))
    if ws is not None:
        ws.fill_(float("nan"))
    dqt.dqt_attn_fwd(a, Qd, Kd, Vd, O, lse, ws)
    torch.cuda.synchronize()
    ref = R.attention(Q, K, V, qs, ks, d ** -0.5 if scale is None else scale, causal, dO if train else None)
    own_q = torch.zeros(tq, dtype=torch.bool)
    own_q[qs[0]:qs[-1]] = True
    own_k = torch.zeros(tk, dtype=torch.bool)
    own_k[ks[0]:ks[-1]] = True
    close("O", O[own_q], ref["O"][own_q], ref["t_O"][own_q])
    close("lse", lse[:, own_q], ref["lse"][:, own_q], ref["t_lse"][:, own_q])
    assert (O[~own_q] == SENT).all() and (lse[:, ~own_q] == SENT).all()
    if not train:
        return
    dQ, dK, dV = like(Qd), like(Kd), like(Vd)
    ws = dqt.workspace(dqt.dqt_attn_bwd_workspace(a))
    if ws is not None:
        ws.fill_(float("nan"))
    dqt.dqt_attn_bwd(a, Qd, Kd, Vd, O, lse, dOd, dQ, dK, dV, ws)
    torch.cuda.synchronize()
    for n, got, own in (("dQ", dQ, own_q), ("dK", dK, own_k), ("dV", dV, own_k)):
        close(n, got[own], ref[n][own], ref["t_" + n][own])
        assert (got[~own] == SENT).all(), n
        if ref[n][own].norm() > 0:
            err = (got[own].double().cpu() - ref[n][own]).norm() / ref[n][own].norm()
            assert err < 1.5 * R.BF16, (n, float(err))


LENGTHS = [
    # (query lengths, key lengths)
    ([1], [1]),
    ([37], [37]),
    ([64, 65, 1, 63], [64, 65, 1, 63]),
    ([127, 128, 129], [127, 128, 129]),
    ([300, 0, 17, 0], [300, 0, 17, 0]),
    ([1, 1, 1, 1, 1, 1], [1, 2, 63, 64, 65, 1000]),             # new tokens
    ([40, 3, 200, 130], [100, 500, 231, 129]),                  # chunks; the last one's first query sees nothing
    ([50, 10, 0], [7, 0, 30]),                                  # rows that see nothing; no keys; no queries
]


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("li", range(len(LENGTHS)))
@pytest.mark.parametrize("heads,kvh", [(2, 2), (6, 2), (8, 1)])
def test_attention_matches_float64(lib, d, li, heads, kvh):
    lq, lk = LENGTHS[li]
    log(f"attention d={d} heads={heads}/{kvh} lq={lq} lk={lk}")
    run(d, heads, kvh, lq, lk, seed=li)


@pytest.mark.parametrize("d", [64, 128])
def test_attention_without_mask(lib, d):
    log(f"attention not causal d={d}")
    run(d, 4, 2, [1, 70, 129, 0], [200, 3, 129, 5], causal=False, seed=20)


@pytest.mark.parametrize("layout", ["heads", "wide"])
@pytest.mark.parametrize("d", [64, 128])
def test_attention_strides(lib, layout, d):
    log(f"attention layout={layout} d={d}")
    run(d, 6, 3, [33, 100, 1], [90, 100, 300], layout=layout, seed=21)


def test_attention_leaves_other_tokens(lib):
    log("attention: tokens before the first and behind the last sequence")
    run(128, 4, 2, [20, 75], [20, 80], before=13, behind=29, seed=22)
    run(64, 4, 4, [1, 1], [700, 20], before=3, behind=5, seed=23)


def test_attention_many_sequences(lib):
    """More sequences than lanes, empty ones among them."""
    rng = np.random.default_rng(3)
    lq = rng.integers(0, 9, 200).tolist()
    lk = [x + int(c) for x, c in zip(lq, rng.integers(0, 12, 200))]
    log("attention: 200 sequences")
    run(64, 3, 1, lq, lk, seed=24)
    run(128, 2, 2, [1] * 130, rng.integers(1, 40, 130).tolist(), seed=25)


def test_attention_long(lib):
    log("attention: 1 x 2100 of 2 heads, one token over 9001 keys, a chunk over 5000")
    run(128, 2, 1, [2100], [2100], seed=26)
    run(128, 8, 2, [1], [9001], seed=27, train=False)
    run(64, 4, 4, [129], [5000], seed=28)


def test_attention_scale_and_large_scores(lib):
    """Scores of several hundreds: the softmax is nearly one-hot; the running
    maximum moves all along the row."""
    log("attention: large scores")
    run(64, 2, 2, [200], [200], scale=1.0, std=4.0, seed=29, train=False)
    run(128, 2, 1, [90], [150], scale=0.01, seed=30)


def test_attention_one_sequence_without_starts(lib):
    gen = torch.Generator().manual_seed(5)
    Q, Qd = tensors(gen, 77, 4, 64, "plain")
    K, Kd = tensors(gen, 77, 2, 64, "plain")
    V, Vd = tensors(gen, 77, 2, 64, "plain")
    log("attention without starts")
    a = dqt.attn(77, 77, 4, 2, 64)
    O = torch.empty_like(Qd)
    dqt.dqt_attn_fwd(a, Qd, Kd, Vd, O)           # (no lse)
    torch.cuda.synchronize()
    ref = R.attention(Q, K, V, [0, 77], [0, 77], 0.125, True)
    close("O", O, ref["O"], ref["t_O"])


def test_attention_infinite_scores_stay_in_their_sequence(lib):
    """A sequence of infinities and NaN leaves the next one's results alone."""
    gen = torch.Generator().manual_seed(6)
    lens = [40, 100, 30]
    s = starts(lens)
    T = int(s[-1])
    Q, Qd = tensors(gen, T, 2, 128, "plain")
    K, Kd = tensors(gen, T, 2, 128, "plain")
    V, Vd = tensors(gen, T, 2, 128, "plain")
    G, Gd = tensors(gen, T, 2, 128, "plain", 1e-2)
    st = torch.from_numpy(s.astype(np.int32)).to(DEV)
    a = dqt.attn(T, T, 2, 2, 128, st, st)
    ws = dqt.workspace(dqt.dqt_attn_bwd_workspace(a))

    def both(q, k, v):
        O, lse = torch.empty_like(q), torch.empty((2, T), dtype=torch.float32, device=DEV)
        g = [torch.empty_like(q) for _ in range(3)]
        dqt.dqt_attn_fwd(a, q, k, v, O, lse, dqt.workspace(dqt.dqt_attn_fwd_workspace(a)))
        dqt.dqt_attn_bwd(a, q, k, v, O, lse, Gd, *g, ws)
        torch.cuda.synchronize()
        return [O, *g]

    log("attention: non-finite neighbours")
    good = both(Qd, Kd, Vd)
    for t in (Qd, Kd, Vd):
        t[s[1]:s[2]] = float("nan")
        t[s[1] + 3] = float("inf")
    bad = both(Qd, Kd, Vd)
    for x, y in zip(good, bad):
        for i in (0, 2):
            assert torch.equal(x[s[i]:s[i + 1]], y[s[i]:s[i + 1]])


def test_attention_gradient_against_differences(lib):
    """The kernels' gradients along random directions against central
    differences of the float64 forward (step 1e-4: truncation below 1e-7)."""
    gen = torch.Generator().manual_seed(7)
    lq, lk, heads, kvh, d = [33, 5], [40, 77], 4, 2, 64
    qs, ks = starts(lq), starts(lk)
    Q, Qd = tensors(gen, 38, heads, d, "plain")
    K, Kd = tensors(gen, 117, kvh, d, "plain")
    V, Vd = tensors(gen, 117, kvh, d, "plain")
    dO, dOd = tensors(gen, 38, heads, d, "plain")
    st = [torch.from_numpy(x.astype(np.int32)).to(DEV) for x in (qs, ks)]
    a = dqt.attn(38, 117, heads, kvh, d, *st)
    O, lse = torch.empty_like(Qd), torch.empty((heads, 38), dtype=torch.float32, device=DEV)
    g = [torch.empty_like(t) for t in (Qd, Kd, Vd)]
    log("attention: differences")
    dqt.dqt_attn_fwd(a, Qd, Kd, Vd, O, lse, dqt.workspace(dqt.dqt_attn_fwd_workspace(a)))
    dqt.dqt_attn_bwd(a, Qd, Kd, Vd, O, lse, dOd, *g, dqt.workspace(dqt.dqt_attn_bwd_workspace(a)))
    torch.cuda.synchronize()
    ref = R.attention(Q, K, V, qs, ks, 0.125, True, dO)
    base = [t.double() for t in (Q, K, V)]
    for i, n in enumerate(("dQ", "dK", "dV")):
        r = torch.randn(base[i].shape, generator=gen, dtype=torch.float64)

        def loss(h):
            x = [b + (h * r if j == i else 0) for j, b in enumerate(base)]
            return float((R.attention(*x, qs, ks, 0.125, True)["O"] * dO.double()).sum())

        diff = (loss(1e-4) - loss(-1e-4)) / 2e-4
        got = float((g[i].double().cpu() * r).sum())
        tol = float((ref["t_" + n] * r.abs()).sum()) + 1e-5 * abs(diff)
        assert abs(got - diff) <= tol, (n, got, diff, tol)


# one block's rows shared by two groups of waves; 64-wide heads; rows of few
# key heads split in the backward
@pytest.mark.parametrize("lens,heads,kvh,d", [([700, 33, 260], 8, 2, 128), ([700, 33, 260], 8, 2, 64),
                                              ([1500, 800], 8, 1, 64), ([1000], 4, 4, 128)])
def test_attention_is_reproducible_and_streams(lib, lens, heads, kvh, d):
    """The same bits on every call, on two streams at once (a workspace each)."""
    gen = torch.Generator().manual_seed(8)
    T = sum(lens)
    st = torch.from_numpy(starts(lens).astype(np.int32)).to(DEV)
    _, Qd = tensors(gen, T, heads, d, "plain")
    _, Kd = tensors(gen, T, kvh, d, "plain")
    _, Vd = tensors(gen, T, kvh, d, "plain")
    _, Gd = tensors(gen, T, heads, d, "plain")
    a = dqt.attn(T, T, heads, kvh, d, st, st)

    def bufs():
        return dict(O=torch.empty_like(Qd), lse=torch.empty((heads, T), dtype=torch.float32, device=DEV),
                    dQ=torch.empty_like(Qd), dK=torch.empty_like(Kd), dV=torch.empty_like(Vd),
                    f=dqt.workspace(dqt.dqt_attn_fwd_workspace(a)), b=dqt.workspace(dqt.dqt_attn_bwd_workspace(a)))

    def go(b, stream=None):
        dqt.dqt_attn_fwd(a, Qd, Kd, Vd, b["O"], b["lse"], b["f"], stream=stream)
        dqt.dqt_attn_bwd(a, Qd, Kd, Vd, b["O"], b["lse"], Gd, b["dQ"], b["dK"], b["dV"], b["b"], stream=stream)

    log(f"attention: two streams {lens} {heads}/{kvh} d={d}")
    first, x, y = bufs(), bufs(), bufs()
    go(first)
    torch.cuda.synchronize()
    s1, s2 = torch.cuda.Stream(), torch.cuda.Stream()
    for _ in range(4):
        go(x, s1)
        go(y, s2)
        torch.cuda.synchronize()
        for b in (x, y):
            for k in ("O", "lse", "dQ", "dK", "dV"):
                assert torch.equal(first[k], b[k]), k


@pytest.mark.parametrize("lens,heads,kvh,d", [([1500, 800], 8, 1, 64), ([900, 1100], 6, 2, 128)])
def test_attention_split_rows_of_the_backward(lib, lens, heads, kvh, d):
    """Few key heads: dk and dv of a key tile are formed by several blocks."""
    log(f"attention: split rows {lens} {heads}/{kvh} d={d}")
    T = sum(lens)
    a = dqt.attn(T, T, heads, kvh, d, torch.zeros(len(lens) + 1, dtype=torch.int32, device=DEV),
                 torch.zeros(len(lens) + 1, dtype=torch.int32, device=DEV))
    assert dqt.dqt_attn_bwd_workspace(a) > 8 * T * heads
    run(d, heads, kvh, lens, lens, seed=31, before=2, behind=3)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("heads,kvh", [(12, 12), (30, 30), (16, 8)])
def test_attention_blocks_of_one_and_two_groups(lib, heads, kvh, d):
    """Numbers of blocks on both sides of the rules for two groups of waves
    per block and for split rows, with lengths of odd numbers of tiles."""
    log(f"attention: groups of waves, {heads}/{kvh} heads d={d}")
    run(d, heads, kvh, [1217, 1, 640], [1217, 1, 640], seed=32, before=1, behind=2)


@pytest.mark.parametrize("d", [64, 128])
def test_attention_many_long_sequences(lib, d):
    """More sequences than lanes, of up to several tiles, and keys that queries
    of any position see."""
    rng = np.random.default_rng(4)
    lens = rng.integers(0, 640, 70).tolist()
    log(f"attention: 70 sequences of up to 640 tokens d={d}")
    run(d, 2, 1, lens, lens, seed=33, behind=4)
    run(d, 9, 9, [700, 130, 1], [300, 900, 500], causal=False, seed=34)


def test_attention_starts_out_of_range_stay_in_the_tensors(lib):
    """Starts that break the rules give wrong results but touch nothing outside:
    they are clamped to the tensors, and descending ones are empty."""
    T, heads, kvh, d, pad = 300, 4, 2, 64, 64
    gen = torch.Generator().manual_seed(35)

    def inner(n, fill):
        buf = torch.full((T + 2 * pad, n, d), fill, dtype=torch.bfloat16, device=DEV)
        return buf, buf[pad:pad + T]

    ins = [inner(n, 0.0) for n in (heads, kvh, kvh, heads)]
    for _, x in ins:
        x.copy_(torch.randn(x.shape, generator=gen).to(torch.bfloat16))
    for bad in ([0, 500, 900, 300], [-70, 40, 20, 290], [250, 100, 400, -5], [300, 300, 300, 301]):
        log(f"attention: starts {bad}")
        st = torch.tensor(bad, dtype=torch.int32, device=DEV)
        a = dqt.attn(T, T, heads, kvh, d, st, st)
        outs = [inner(n, SENT) for n in (heads, heads, kvh, kvh)]
        lse = torch.zeros((heads, T), dtype=torch.float32, device=DEV)
        q, k, v, do = (x for _, x in ins)
        o, dq, dk, dv = (x for _, x in outs)
        ws = dqt.workspace(max(dqt.dqt_attn_fwd_workspace(a), dqt.dqt_attn_bwd_workspace(a)))
        dqt.dqt_attn_fwd(a, q, k, v, o, lse, ws)
        dqt.dqt_attn_bwd(a, q, k, v, o, lse, do, dq, dk, dv, ws)
        torch.cuda.synchronize()
        for buf, _ in outs:
            assert (buf[:pad] == SENT).all() and (buf[pad + T:] == SENT).all()


def test_attention_offsets_past_32_bits(lib):
    """Sequences at the end of 5 GB of keys and of values, and of 5 GB of
    queries: the bits of the same call on copies at the start."""
    log("attention: long tensors")
    gen = torch.Generator(device=DEV).manual_seed(9)
    tk, kvh, d = 2_500_000, 8, 128
    K, V, O = (torch.empty((tk, kvh, d), dtype=torch.bfloat16, device=DEV) for _ in range(3))
    lens = [700, 300]
    n = sum(lens)
    for t in (K, V):
        t[-n:] = torch.randn((n, kvh, d), generator=gen, device=DEV).to(torch.bfloat16)
    Q = torch.empty((tk, kvh, d), dtype=torch.bfloat16, device=DEV)
    Q[-n:] = torch.randn((n, kvh, d), generator=gen, device=DEV).to(torch.bfloat16)
    G = Q * 0.01

    def both(q, k, v, o, g, s):
        st = torch.tensor(s, dtype=torch.int32, device=DEV)
        T = q.shape[0]
        a = dqt.attn(T, T, kvh, kvh, d, st, st)
        lse = torch.empty((kvh, T), dtype=torch.float32, device=DEV)
        out = [torch.empty_like(q) for _ in range(3)]
        dqt.dqt_attn_fwd(a, q, k, v, o, lse, dqt.workspace(dqt.dqt_attn_fwd_workspace(a)))
        dqt.dqt_attn_bwd(a, q, k, v, o, lse, g, *out, dqt.workspace(dqt.dqt_attn_bwd_workspace(a)))
        torch.cuda.synchronize()
        return [x[-n:].clone() for x in (o, *out)] + [lse[:, -n:].clone()]

    far = both(Q, K, V, O, G, [tk - n, tk - n + lens[0], tk])
    small = [t[-n:].clone() for t in (Q, K, V, O, G)]
    near = both(*small, [0, lens[0], n])
    for x, y in zip(far, near):
        assert x.isfinite().all() and (x - y).abs().max() <= 2.0 ** -6 * y.abs().max()


@pytest.mark.parametrize("tk", [(1 << 31) - 129, (1 << 31) - 2000, (1 << 30) + 7])
def test_attention_over_the_largest_number_of_keys(lib, tk):
    """One new token over as many keys as a call takes, all of them one row of
    memory (token stride 0).  With q = 0 every key counts alike: o = v, and lse =
    log tk shows that none is lost (one split's share would move it by 6e-4).  v
    are powers of two, so that the sums are exact."""
    log(f"attention: {tk} keys")
    heads, d = 2, 64
    gen = torch.Generator().manual_seed(36)
    K = torch.randn((1, 1, d), generator=gen).to(torch.bfloat16).to(DEV)
    V = (2.0 ** torch.randint(-3, 4, (1, 1, d), generator=gen) * (torch.randint(0, 2, (1, 1, d), generator=gen) * 2 - 1))
    V = V.to(torch.bfloat16).to(DEV)
    Q = torch.zeros((1, heads, d), dtype=torch.bfloat16, device=DEV)
    a = dqt.attn(1, tk, heads, 1, d)
    O, lse = torch.full_like(Q, SENT), torch.zeros((heads, 1), dtype=torch.float32, device=DEV)
    n = dqt.dqt_attn_fwd_workspace(a)
    assert n > 0
    ws = dqt.workspace(n)
    ws.fill_(float("nan"))
    dqt.dqt_attn_fwd(a, Q, K.expand(tk, 1, d), V.expand(tk, 1, d), O, lse, ws)
    torch.cuda.synchronize()
    assert torch.equal(O, V.expand(1, heads, d))
    # log2 of a part and of their sum, below 2^5: a few roundings of 2^-19 / 2
    assert (lse.double().cpu() - float(np.log(float(tk)))).abs().max() < 8 * 2.0 ** -20 + 22 * R.F32


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("lq,lk,heads,kvh", [([1, 2, 17, 40], [1, 2, 17, 40], 2, 2), ([64, 33, 128], [64, 33, 128], 4, 2),
                                             ([1, 3, 20, 9], [1, 100, 128, 65], 8, 1)])
@pytest.mark.parametrize("causal", [True, False])
def test_attention_gradients_of_few_keys_do_not_take_delta_from_o(lib, d, lq, lk, heads, kvh, causal):
    """Rows of at most 128 keys: do.o is found from p and v, not from the bf16 O,
    whose error would count beside do.v - do.o.  O handed to the backward is off
    by 2 % of its largest value at random, and dQ, dK stay what p and g in bf16
    and the final rounding allow; taken from that O, do.o would
    move some of them by more (checked below on the reference)."""
    log(f"attention: few keys, O perturbed, d={d} lq={lq} lk={lk} {heads}/{kvh} causal={causal}")
    gen = torch.Generator().manual_seed(40 + d)
    qs, ks = starts(lq), starts(lk)
    Q, Qd = tensors(gen, int(qs[-1]), heads, d, "plain")
    K, Kd = tensors(gen, int(ks[-1]), kvh, d, "plain")
    V, Vd = tensors(gen, int(ks[-1]), kvh, d, "plain")
    dO, dOd = tensors(gen, int(qs[-1]), heads, d, "plain", 1e-2)
    st = [torch.from_numpy(x.astype(np.int32)).to(DEV) for x in (qs, ks)]
    a = dqt.attn(Q.shape[0], K.shape[0], heads, kvh, d, *st, causal=causal)
    O, lse = torch.empty_like(Qd), torch.empty((heads, Q.shape[0]), dtype=torch.float32, device=DEV)
    dqt.dqt_attn_fwd(a, Qd, Kd, Vd, O, lse, dqt.workspace(dqt.dqt_attn_fwd_workspace(a)))
    off = torch.randn(O.shape, generator=gen) * 0.02 * float(O.float().abs().max())
    bent = (O.float().cpu() + off).to(torch.bfloat16)
    g = [torch.empty_like(t) for t in (Qd, Kd, Vd)]
    dqt.dqt_attn_bwd(a, Qd, Kd, Vd, bent.to(DEV), lse, dOd, *g, dqt.workspace(dqt.dqt_attn_bwd_workspace(a)))
    torch.cuda.synchronize()
    # per sequence: exact gradients; what roundings of g (BF16), of p and its
    # exponent (SLACK, on each term of g; where p's sum is off by it, the O that was
    # handed over counts with it) and of the result allow; and the gradients with
    # do.o from that O
    scale, SLACK = d ** -0.5, 2.0 ** -12
    z = dict(dtype=torch.float64)
    want = [torch.zeros(t.shape, **z) for t in (Q, K)]
    tol = [torch.zeros(t.shape, **z) for t in (Q, K)]
    worse = [torch.zeros(t.shape, **z) for t in (Q, K)]
    for s in range(len(lq)):
        A, B = slice(qs[s], qs[s + 1]), slice(ks[s], ks[s + 1])
        see = torch.ones((lq[s], lk[s]), dtype=torch.bool)
        if causal:
            see = torch.arange(lk[s])[None, :] <= torch.arange(lq[s])[:, None] + lk[s] - lq[s]
        for h in range(heads):
            j = h // (heads // kvh)
            q, k, v, do = Q[A, h].double(), K[B, j].double(), V[B, j].double(), dO[A, h].double()
            p = torch.softmax((scale * q @ k.T).masked_fill(~see, -np.inf), 1)
            dp = do @ v.T
            mag = do.abs() @ v.abs().T
            ds = p * (dp - (p * dp).sum(1, keepdim=True))
            ob = bent[A, h].double()
            t_ds = R.BF16 * ds.abs() + SLACK * p * (mag + (p * mag).sum(1, keepdim=True)
                                                    + (do * ob).abs().sum(1, keepdim=True))
            bad = p * (dp - (do * ob).sum(1, keepdim=True))
            want[0][A, h], tol[0][A, h], worse[0][A, h] = scale * ds @ k, scale * t_ds @ k.abs(), scale * bad @ k
            want[1][B, j] += scale * ds.T @ q
            tol[1][B, j] += scale * t_ds.T @ q.abs()
            worse[1][B, j] += scale * bad.T @ q
    for n, got, w, t, o in zip(("dQ", "dK"), g, want, tol, worse):
        t = t + R.BF16 * w.abs() * (1 + 2.0 ** -7)
        close(n, got, w, t)
        assert ((o - w).abs() > t).double().mean() > 0.03, n


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("heads,kvh", [(5, 1), (14, 2), (96, 1), (130, 2), (1024, 1)])
def test_attention_odd_and_large_groups(lib, heads, kvh, d):
    """Groups that do not divide a tile of rows, or fill several by themselves."""
    log(f"attention: groups of {heads // kvh} d={d}")
    lq, lk = ([9, 1, 30], [9, 40, 31]) if heads < 1000 else ([3, 1], [5, 70])
    run(d, heads, kvh, lq, lk, seed=37, before=1, behind=1)


def call(a, q, k, v, do):
    """Forward and backward: [O, lse, dQ, dK, dV]."""
    tq, heads = q.shape[:2]
    new = lambda t: torch.full(t.shape, SENT, dtype=torch.bfloat16, device=DEV)
    O, lse, g = new(q), torch.full((heads, tq), SENT, dtype=torch.float32, device=DEV), [new(t) for t in (q, k, v)]
    dqt.dqt_attn_fwd(a, q, k, v, O, lse, dqt.workspace(dqt.dqt_attn_fwd_workspace(a)))
    dqt.dqt_attn_bwd(a, q, k, v, O, lse, do, *g, dqt.workspace(dqt.dqt_attn_bwd_workspace(a)))
    torch.cuda.synchronize()
    return [O, lse, *g]


@pytest.mark.parametrize("d", [64, 128])
def test_attention_inputs_of_stride_zero(lib, d):
    """Heads or tokens that share memory give the bits of their copies."""
    gen = torch.Generator(device=DEV).manual_seed(38)
    r = lambda *s: torch.randn(s, generator=gen, device=DEV).to(torch.bfloat16)
    T, heads, kvh = 200, 6, 3
    st = torch.tensor([0, 70, 200], dtype=torch.int32, device=DEV)
    a = dqt.attn(T, T, heads, kvh, d, st, st)
    q, k, v, do = r(T, 1, d), r(T, 1, d), r(1, kvh, d), r(T, heads, d)
    views = [q.expand(T, heads, d), k.expand(T, kvh, d), v.expand(T, kvh, d), do[:1].expand(T, heads, d)]
    log(f"attention: inputs of stride zero d={d}")
    for x, y in zip(call(a, *views), call(a, *[t.contiguous() for t in views])):
        assert torch.equal(x, y)


def test_attention_one_start_alone(lib):
    """Starts of the queries or of the keys alone: the other is all tokens."""
    gen = torch.Generator(device=DEV).manual_seed(39)
    r = lambda *s: torch.randn(s, generator=gen, device=DEV).to(torch.bfloat16)
    q, k, v, do = r(50, 4, 64), r(90, 2, 64), r(90, 2, 64), r(50, 4, 64)
    s = lambda *x: torch.tensor(x, dtype=torch.int32, device=DEV)
    log("attention: one start alone")
    want = call(dqt.attn(50, 90, 4, 2, 64, s(0, 50), s(0, 90)), q, k, v, do)
    for qs, ks in ((s(0, 50), None), (None, s(0, 90)), (None, None)):
        for x, y in zip(call(dqt.attn(50, 90, 4, 2, 64, qs, ks), q, k, v, do), want):
            assert torch.equal(x, y)


@pytest.mark.parametrize("d", [64, 128])
def test_attention_without_queries_or_keys(lib, d):
    """No key: O and dQ 0, lse -inf.  No query: dK and dV 0."""
    e, x = (torch.ones((n, 2, d), dtype=torch.bfloat16, device=DEV) for n in (0, 140))
    log(f"attention: no queries, no keys d={d}")
    O, lse, dQ, dK, dV = call(dqt.attn(140, 0, 2, 2, d), x, e, e, x)
    assert (O == 0).all() and (dQ == 0).all() and (lse == -float("inf")).all() and dK.numel() == dV.numel() == 0
    O, lse, dQ, dK, dV = call(dqt.attn(0, 140, 2, 2, d), e, x, x, e)
    assert (dK == 0).all() and (dV == 0).all() and O.numel() == lse.numel() == dQ.numel() == 0
