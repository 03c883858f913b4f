"""Token log probabilities, entropy, alternatives and the logits' gradient
against plain float64 arithmetic."""
import numpy as np
import pytest
import torch

import op_reference as R
from gpu_util import DEV, log
from paper_2412_04787_amd import dqt

pytestmark = pytest.mark.gpu

INF = float("inf")


def forward(X, t, top=0, ent=True):
    M, V = X.shape
    f = lambda *s: torch.full(s, 777.0, dtype=torch.float32, device=DEV)
    o = dict(logp=f(M), lse=f(M), entropy=f(M) if ent else None, stat=f(M, 2),
             ids=torch.full((M, top), -7, dtype=torch.int64, device=DEV) if top else None, tl=f(M, top) if top else None)
    ws = dqt.workspace(dqt.dqt_logprob_workspace(M, V, top))
    if ws is not None:
        ws.fill_(float("nan"))
    dqt.dqt_logprob_fwd(X, t, o["logp"], o["lse"], o["entropy"], o["stat"], o["ids"], o["tl"], ws)
    torch.cuda.synchronize()
    return o


def check(X, Xd, t, top, ent=True):
    """X: the values on the host (fp32), Xd: the device tensor."""
    V = X.shape[1]
    o = forward(Xd, t.to(DEV), top, ent)
    ref = R.logprob(X, t)
    for n in ("lse", "logp") + (("entropy",) if ent else ()):
        got = o[n].double().cpu()
        bad = ~((got - ref[n]).abs() <= ref["t_" + n]) & (got != ref[n])
        assert not bad.any(), (n, got[bad][:4], ref[n][bad][:4])
    if top:
        val, idx = torch.sort(X, dim=1, descending=True, stable=True)
        assert torch.equal(o["ids"].cpu(), idx[:, :top]), "top ids"
        want = ref["d"].gather(1, idx[:, :top])
        want[torch.isinf(val[:, :top])] = -INF
        got = o["tl"].double().cpu()
        tol = ref["t_d"] + 2 * R.F32 * torch.nan_to_num(want.abs(), posinf=0)
        assert (((got - want).abs() <= tol) | (got == want)).all()
    return o, ref


def logits(M, V, dt, seed, masked=True):
    g = torch.Generator().manual_seed(seed)
    X = torch.randn((M, V), generator=g) * 2
    if masked and V > 3:
        X[:, V - max(1, V // 64):] = -INF
        X[M // 2, V // 2:] = -INF
    X = X.to(dt)
    t = torch.randint(0, max(1, V // 2), (M,), generator=g)
    if M > 2:
        t[1] = -100
        t[2] = V
    return X, t


SIZES = [(1, 1), (2, 2), (5, 7), (3, 100), (17, 1000), (300, 1001), (4, 4096), (1, 8192), (3, 32000), (1, 128001),
         (600, 4099)]


@pytest.mark.parametrize("dt", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("top", [0, 1, 5, 32])
@pytest.mark.parametrize("M,V", SIZES)
def test_logprob_forward(lib, dt, top, M, V):
    top = min(top, V)
    log(f"logprob M={M} V={V} top={top} {dt}")
    X, t = logits(M, V, dt, V + top)
    check(X.float(), X.to(DEV), t, top, ent=top != 1)


@pytest.mark.parametrize("dt", [torch.bfloat16, torch.float32])
def test_logprob_strided_rows(lib, dt):
    """Rows at every alignment, of a wider buffer."""
    for pad in (1, 2, 3, 5, 8):
        log(f"logprob stride {pad} {dt}")
        X, t = logits(9, 517, dt, pad)
        buf = torch.full((9, 517 + pad), 100.0, dtype=dt, device=DEV)
        buf[:, :517] = X.to(DEV)
        check(X.float(), buf[:, :517], t, 4)


@pytest.mark.parametrize("dt", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("M", [3, 530])
def test_logprob_ties_and_masked_rows(lib, dt, M):
    """Constant rows, rows of few distinct values, rows with fewer finite
    logits than alternatives, rows of nothing but -inf, the lowest finite value."""
    log(f"logprob ties {dt} M={M}")
    V = 9000
    X = torch.zeros((M, V))
    X[1] = (torch.arange(V) % 3).float()
    X[2] = -INF
    X[2, 4000] = 1.5
    X[2, 17] = 1.5
    if M > 3:
        X[3] = -INF
        X[4] = float(torch.finfo(dt).min)
        X[5, ::2] = float(torch.finfo(dt).min)
        X[6] = torch.arange(V).float()
        X[7] = -torch.arange(V).float()
    X = X.to(dt)
    t = torch.zeros((M,), dtype=torch.int64)
    t[2] = 17
    check(X.float(), X.to(DEV), t, 32)


@pytest.mark.parametrize("dt", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("V", [61439, 61440, 70001])
def test_logprob_split_rows(lib, dt, V):
    """Rows on both sides of the length from which several blocks share one:
    ties over all of them, masks that leave a block or a row nothing, rows of
    another stride."""
    M = 8
    log(f"logprob split rows V={V} {dt}")
    X = torch.randn((M, V), generator=torch.Generator().manual_seed(V))
    X[1] = (torch.arange(V) % 3).float()
    X[2] = -INF
    X[2, V - 1] = 1.5
    X[2, 17] = 1.5
    X[3] = -INF
    X[4] = float(torch.finfo(dt).min)
    X[5, :V // 2] = -INF
    X[6] = torch.arange(V).float()
    X[7] = -torch.arange(V).float()
    X = X.to(dt)
    t = torch.tensor([V - 1, 0, 17, 3, 5, V // 2, V - 1, -1])
    buf = torch.full((M, V + 3), 50.0, dtype=dt, device=DEV)
    view = buf[:, :V]
    view.copy_(X)
    check(X.float(), view, t, 32)


@pytest.mark.parametrize("M", [1, 600])
def test_logprob_alternatives_of_adverse_rows(lib, M):
    """The largest logits all lie where few threads read them: more candidates
    reach the bound than LDS holds."""
    log(f"logprob adverse rows M={M}")
    V = 65536
    g = torch.Generator().manual_seed(4)
    X = torch.rand((M, V), generator=g)
    piece = (torch.arange(V) // 4) % 256
    X[:, piece < 80] += 5.0
    check(X, X.to(DEV), torch.zeros((M,), dtype=torch.int64), 20)


def test_logprob_non_finite_rows(lib):
    """NaN and +inf reach their own row's results alone; alternatives stay
    distinct tokens."""
    log("logprob non-finite rows")
    X, t = logits(6, 3000, torch.float32, 11)
    clean = forward(X.to(DEV), t.to(DEV), 8)
    Y = X.clone()
    Y[0, 5] = float("nan")
    Y[1] = float("nan")
    Y[3, 9] = INF
    Y[3, 10] = INF
    Y[4, 70] = -float("nan")
    got = forward(Y.to(DEV), t.to(DEV), 8)
    for r in (0, 1, 3, 4):
        assert torch.isnan(got["lse"][r]) and torch.isnan(got["entropy"][r])
        ids = got["ids"][r].tolist()
        assert len(set(ids)) == 8 and all(0 <= i < 3000 for i in ids)
    for r in (2, 5):
        for n in ("lse", "logp", "entropy", "ids", "tl"):
            assert torch.equal(got[n][r], clean[n][r])


@pytest.mark.parametrize("dt", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("ent", [True, False])
@pytest.mark.parametrize("M,V,pad", [(1, 1, 0), (5, 7, 0), (17, 1000, 0), (33, 1001, 0), (4, 32000, 0), (3, 20000, 3)])
def test_logprob_backward(lib, dt, ent, M, V, pad):
    log(f"logprob backward M={M} V={V} pad={pad} {dt} entropy={ent}")
    X, t = logits(M, V, dt, V + 1)
    if M > 3:
        X[3] = -INF                      # a row without a finite logit
        X[0] = float(torch.finfo(dt).min)    # all equal: p = 1 / V, whatever the value
    Xd = torch.zeros((M, V + pad), dtype=dt, device=DEV)[:, :V]
    Xd.copy_(X)
    g = torch.Generator().manual_seed(2)
    dl, de = torch.randn((M,), generator=g), torch.randn((M,), generator=g) * 0.1
    o = forward(Xd, t.to(DEV))
    ref = R.logprob(X.float(), t)
    buf = torch.full((M, V + 5), 3.0, dtype=dt, device=DEV)      # (another stride: other alignments)
    dX = buf[:, :V]
    args = (t.to(DEV), o["stat"], dl.to(DEV))
    kw = dict(entropy=o["entropy"], dent=de.to(DEV)) if ent else {}
    dqt.dqt_logprob_bwd(Xd, *args, dX, **kw)
    same = Xd.clone() if pad == 0 else torch.zeros((M, V + pad), dtype=dt, device=DEV)[:, :V].copy_(Xd)
    dqt.dqt_logprob_bwd(same, *args, same, **kw)                 # in place
    torch.cuda.synchronize()
    assert torch.equal(same, dX) and (buf[:, V:] == 3.0).all()
    gl = torch.where(ref["has"], dl.double(), torch.zeros(M, dtype=torch.float64))[:, None]
    pick = torch.nn.functional.one_hot(t.clamp(0, V - 1), V).double() * ref["has"][:, None]
    some = torch.isfinite(ref["lse"])[:, None]
    want = torch.where(some, gl * (pick - ref["p"]), torch.zeros_like(ref["p"]))
    e = de.double()[:, None] if ent else torch.zeros((M, 1), dtype=torch.float64)
    want = want - torch.where(some, e * (ref["plogp"] + ref["p"] * ref["entropy"][:, None]), torch.zeros_like(want))
    # p: the error of lse and of one exponent below 2^7; entropy's own; then 6 roundings
    rel = torch.where(some, torch.full_like(some, ref["t_d"] + 128 * R.F32, dtype=torch.float64), torch.zeros_like(some, dtype=torch.float64))
    terms = gl.abs() * pick + ref["p"] * (gl.abs() + e.abs() * (ref["entropy"].abs()[:, None] + 1)) + e.abs() * ref["plogp"].abs()
    tol = (rel + 8 * R.F32) * terms + e.abs() * ref["p"] * torch.nan_to_num(ref["t_entropy"])[:, None]
    half = R.BF16 if dt == torch.bfloat16 else R.F32
    tol = tol + half * want.abs() * (1 + 2.0 ** -7) + 1e-37
    err = (dX.double().cpu() - want).abs()
    assert (err <= tol).all(), (float(err.max()), int((err > tol).sum()))


def test_logprob_gradient_against_differences(lib):
    M, V = 3, 50
    X, t = logits(M, V, torch.float32, 5, masked=False)
    t = torch.tensor([3, 0, 49])
    dl, de = torch.tensor([1.0, -0.5, 2.0]), torch.tensor([0.3, 0.2, -0.7])
    o = forward(X.to(DEV), t.to(DEV))
    dX = torch.empty((M, V), dtype=torch.float32, device=DEV)
    log("logprob: differences")
    dqt.dqt_logprob_bwd(X.to(DEV), t.to(DEV), o["stat"], dl.to(DEV), dX, o["entropy"], de.to(DEV))
    torch.cuda.synchronize()
    h = 1e-5
    for j in range(V):
        Y = X.double()
        up, down = Y.clone(), Y.clone()
        up[:, j] += h
        down[:, j] -= h
        a, b = R.logprob(up, t), R.logprob(down, t)
        diff = (dl.double() * (a["logp"] - b["logp"]) + de.double() * (a["entropy"] - b["entropy"])) / (2 * h)
        assert ((dX[:, j].double().cpu() - diff).abs() <= 2e-6 * (1 + diff.abs())).all()


def test_logprob_more_rows_than_blocks(lib):
    """Rows past the largest grid of the gradient give what they give alone."""
    M, V, tail = 1_050_001, 9, 3000
    X = torch.randn((M, V), generator=torch.Generator().manual_seed(12)).to(torch.bfloat16).to(DEV)
    t = (torch.arange(M, device=DEV) % 11) - 1
    g = torch.linspace(-1, 1, M, device=DEV)
    log("logprob: 1050001 rows")

    def go(x, t, g):
        o = forward(x, t)
        dX = torch.empty_like(x)
        dqt.dqt_logprob_bwd(x, t, o["stat"], g, dX, o["entropy"], g)
        torch.cuda.synchronize()
        return [o["logp"], o["lse"], o["entropy"], dX]

    # (the tail's rows as a tensor of their own: their alignment differs, not their values)
    for x, y in zip(go(X, t, g), go(X[-tail:].clone(), t[-tail:].clone(), g[-tail:].clone())):
        assert (x[-tail:].float() - y.float()).abs().max() <= 2.0 ** -7 * y.float().abs().max()


def test_logprob_empty(lib):
    e = torch.empty((0, 10), device=DEV)
    v = torch.empty((0,), device=DEV)
    dqt.dqt_logprob_fwd(e, v.long(), v, v)
    dqt.dqt_logprob_bwd(e, v.long(), torch.empty((0, 2), device=DEV), v, e)


def zeros_of_both_signs(M, V, dt):
    """Rows whose largest logits are zeros of either sign: ties over the k-th
    place, in one thread's piece and far apart."""
    X = torch.full((M, V), -1.0)
    X[0, :3] = torch.tensor([-0.0, 0.0, -1.0])
    X[1] = torch.where(torch.arange(V) % 2 == 0, -0.0, 0.0)
    X[2] = torch.where(torch.arange(V) < V // 2, -0.0, 0.0)
    X[3, V - 1] = 0.0
    X[3, 7] = -0.0
    X[3, V // 2] = 2.0
    X[4] = -0.0
    X[4, V - 2] = 0.0
    X[5, ::3] = -0.0
    X[5, 1::3] = 0.0
    X[5, 5] = 1e-30
    X[5, 6] = -1e-30
    return X.to(dt)


@pytest.mark.parametrize("dt", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("V", [9, 1000, 9000, 70001])
def test_logprob_zeros_of_either_sign_are_equal(lib, dt, V):
    """The lower id comes first among them, in one block's row and in split rows."""
    X = zeros_of_both_signs(6, V, dt)
    t = torch.tensor([0, 1, V - 1, 7, V - 2, 0])
    for top in (1, 2, 5, min(V, 32)):
        log(f"logprob zeros of either sign V={V} top={top} {dt}")
        check(X.float(), X.to(DEV), t, top)


def gradient(X, t, dl, de=None):
    o = forward(X, t)
    dX = torch.full_like(X, 5.0)
    kw = {} if de is None else dict(entropy=o["entropy"], dent=de)
    dqt.dqt_logprob_bwd(X, t, o["stat"], dl, dX, **kw)
    torch.cuda.synchronize()
    return dX


@pytest.mark.parametrize("dt", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("ent", [False, True])
@pytest.mark.parametrize("V", [40, 3000, 70001])
def test_logprob_gradient_of_non_finite_rows(lib, dt, ent, V):
    """A row with a NaN or +inf has no finite gradient, whatever else it holds:
    one NaN, NaN alone, NaN and -inf, +inf.  A row of -inf alone gets 0, and
    the other rows what they get without such neighbours."""
    log(f"logprob gradient of non-finite rows V={V} {dt} entropy={ent}")
    X, _ = logits(7, V, dt, V + 3, masked=False)
    t = torch.tensor([3, 0, 5, V - 1, 2, 7, 8]).to(DEV)
    dl = torch.linspace(-1.5, 1.0, 7).to(DEV)
    de = torch.linspace(0.1, 0.7, 7).to(DEV) if ent else None
    clean = gradient(X.to(DEV), t, dl, de)
    Y = X.clone()
    Y[0, V // 2] = float("nan")
    Y[1] = float("nan")
    Y[2] = -INF
    Y[2, V - 2] = float("nan")
    Y[3, 11] = INF
    Y[4] = -INF
    got = gradient(Y.to(DEV), t, dl, de)
    for r in (0, 1, 2, 3):
        assert torch.isnan(got[r]).all(), r
    assert (got[4] == 0).all()
    for r in (5, 6):
        assert torch.equal(got[r], clean[r])


@pytest.mark.parametrize("dt", [torch.bfloat16, torch.float32])
def test_logprob_gradient_of_padding(lib, dt):
    """A row without a target has the gradient 0, whatever its logits are; its
    entropy's gradient still counts where that is asked for."""
    log(f"logprob gradient of padding rows {dt}")
    M, V = 6, 5000
    X, _ = logits(M, V, dt, 41, masked=False)
    X[1] = float("nan")
    X[2, 4] = INF
    X[3] = -INF
    X[4, 9] = float("nan")
    t = torch.tensor([-100, -1, V, V + 7, 2 ** 40, 3]).to(DEV)
    dl = torch.full((M,), -0.25).to(DEV)
    got = gradient(X.to(DEV), t, dl)
    assert (got[:5] == 0).all() and (got[5] != 0).any()
    de = torch.zeros((M,))
    de[0] = 0.5
    both = gradient(X.to(DEV), t, dl, de.to(DEV))
    assert (both[1:5] == 0).all() and torch.isfinite(both[0]).all() and (both[0] != 0).any()


@pytest.mark.parametrize("dt", [torch.bfloat16, torch.float32])
def test_logprob_gradient_of_a_masked_target(lib, dt):
    """A target whose logit is masked: its own column takes g (p is 0 there),
    the others -p g, as the formula says; other masked columns 0."""
    log(f"logprob gradient of a masked target {dt}")
    X = torch.tensor([[0.0, 1.0, -INF, 2.0, -INF, -1.0]]).to(dt)
    t, g = torch.tensor([2]).to(DEV), 0.75
    got = gradient(X.to(DEV), t, torch.tensor([g]).to(DEV)).double().cpu()[0]
    p = torch.softmax(X.double(), 1)[0]
    want = -g * p
    want[2] = g
    half = R.BF16 if dt == torch.bfloat16 else R.F32
    # (p: some 16 fp32 roundings of an exponent of at most 4 and of its sum)
    assert ((got - want).abs() <= (half + 64 * R.F32) * want.abs()).all() and got[4] == 0
    assert float(forward(X.to(DEV), t)["logp"][0]) == -INF


def test_logprob_of_the_largest_vocabulary(lib):
    """A row of 2^28 logits, all zero but a few: sums, alternatives and the
    gradient in closed form."""
    V = 1 << 28
    log("logprob: 2^28 logits")
    X = torch.zeros((1, V), dtype=torch.bfloat16, device=DEV)
    some = {V - 1: 6.0, V - 2: 4.0, 5: 5.0, 1 << 27: 3.0}
    for i, x in some.items():
        X[0, i] = x
    t = torch.tensor([V - 1], device=DEV)
    o = forward(X, t, 6)
    s = V - 4 + sum(np.exp(x) for x in some.values())
    lse, ent = np.log(s), np.log(s) - sum(x * np.exp(x) for x in some.values()) / s
    # (64 blocks of 256 threads sum 2^14 terms of 1 each, exactly up to 2^24)
    assert abs(float(o["lse"][0]) - lse) < 1e-5 and abs(float(o["logp"][0]) - (6.0 - lse)) < 1e-5
    assert abs(float(o["entropy"][0]) - ent) < 1e-4
    assert o["ids"][0].tolist() == [V - 1, 5, V - 2, 1 << 27, 0, 1]
    dX = torch.full_like(X, 7.0)
    dqt.dqt_logprob_bwd(X, t, o["stat"], torch.tensor([1.0], device=DEV), dX)
    torch.cuda.synchronize()
    assert abs(float(dX[0, V - 1]) - (1 - np.exp(6.0) / s)) <= 2.0 ** -8
    for i in (5, V - 2, 1 << 27):
        assert abs(float(dX[0, i]) + np.exp(some[i]) / s) <= 2.0 ** -7 * np.exp(some[i]) / s
    dX[0, list(some)] = dX[0, 0].clone()
    assert (dX == dX[0, 0]).all() and abs(float(dX[0, 0]) * s + 1) <= 2.0 ** -7
