"""Rotary positions (dqt_rope_fwd, dqt_rope_bwd) against a plain float64
implementation: layouts, parts of a head, far and negative positions, strides, in
place; the backward also as the transposed map and against differences."""
import numpy as np
import pytest
import torch

import kv_reference as R
from gpu_util import DEV, log
from paper_2412_04787_amd import dqt

pytestmark = pytest.mark.gpu

SENT = 1.25e4


def make(gen, tokens, heads, d, dt, layout="plain"):
    x = torch.randn((tokens, heads, d), generator=gen).to(dt)
    if layout == "heads":
        return x, x.permute(1, 0, 2).contiguous().to(DEV).permute(1, 0, 2)
    if layout == "wide":
        buf = torch.full((tokens, 3, heads + 1, d + 8), 7.0, dtype=dt)
        buf[:, 1, :heads, :d] = x
        return x, buf.to(DEV)[:, 1, :heads, :d]
    return x, x.to(DEV)


def like(v):
    n = 1 + sum((s - 1) * st for s, st in zip(v.shape, v.stride())) if v.numel() else 0
    return torch.full((n,), SENT, dtype=v.dtype, device=DEV).as_strided(v.shape, v.stride())


def check(got, x, pos, freq, rot, pairs, amp, back):
    ref, t = R.rotate(x, pos, freq, rot, pairs, amp, back)
    if x.dtype is torch.bfloat16:
        t = t + R.BF16 * ref.abs() * (1 + R.BF16)
        t[..., rot:] = 0
    err = (got.double().cpu() - ref).abs()
    assert (err <= t + 1e-37).all(), (float((err - t).max()), (err - t).argmax())


def case(dt, d, rot, pairs, heads, tokens, pos=None, amp=1.0, layout="plain", seed=0, **freqs):
    gen = torch.Generator().manual_seed(seed)
    f = dqt.dqt_rope_freqs(rot, **freqs)
    rope = dqt.rope(d, rot, pairs, amp, **freqs)
    at = np.arange(tokens) if pos is None else np.asarray(pos)
    pd = None if pos is None else torch.tensor(np.asarray(pos), dtype=torch.int32, device=DEV)
    xs = [make(gen, tokens, h, d, dt, layout) for h in heads]
    for fn, back in ((dqt.dqt_rope_fwd, False), (dqt.dqt_rope_bwd, True)):
        ys = [like(x) for _, x in xs]
        fn(rope, [(x, y) for (_, x), y in zip(xs, ys)], pd)
        torch.cuda.synchronize()
        for (x, _), y in zip(xs, ys):
            check(y, x, at, f, rot, pairs, amp, back)
        inplace = [x.clone() if layout == "plain" else x for _, x in xs]
        if layout == "plain":
            fn(rope, [(x, x) for x in inplace], pd)
            torch.cuda.synchronize()
            for x, y in zip(inplace, ys):
                assert torch.equal(x, y)


@pytest.mark.parametrize("dt", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("pairs", [False, True])
@pytest.mark.parametrize("d,rot", [(64, 64), (128, 128), (128, 32), (64, 48), (16, 16), (80, 48), (256, 96)])
def test_rope_matches_float64(lib, dt, pairs, d, rot):
    log(f"rope {dt} d={d} rot={rot} pairs={pairs}")
    rng = np.random.default_rng(d + rot)
    case(dt, d, rot, pairs, [3, 1], 37, rng.integers(0, 5000, 37))
    case(dt, d, rot, pairs, [2], 1)


@pytest.mark.parametrize("pairs", [False, True])
def test_rope_far_positions(lib, pairs):
    """Positions up to 2^31 - 1 and negative ones; stretched contexts."""
    log("rope: far positions")
    pos = [0, 1, -1, 2 ** 31 - 1, -2 ** 31, 10 ** 6 + 3, 131071, 12345678, -77]
    case(torch.float32, 128, 128, pairs, [2, 1], len(pos), pos, seed=1)
    case(torch.float32, 128, 64, pairs, [1], len(pos), pos, amp=1.2079, seed=2, base=500000.0, factor=8.0, context=8192.0,
         slow=1.0, fast=4.0)
    case(torch.bfloat16, 64, 64, pairs, [4], len(pos), pos, seed=3, factor=4.0, slow=0.0, fast=0.0)


@pytest.mark.parametrize("dt", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("layout", ["heads", "wide"])
def test_rope_strides(lib, dt, layout):
    log(f"rope: strides {layout}")
    case(dt, 64, 32, False, [5, 2, 1], 70, np.arange(70) * 3, layout=layout, seed=4)
    case(dt, 128, 128, True, [2, 2, 2, 2], 33, layout=layout, seed=5)


def test_rope_many_tokens_and_empty(lib):
    log("rope: 20000 tokens, none")
    case(torch.bfloat16, 64, 64, False, [2, 1], 20000, seed=6)
    rope = dqt.rope(64)
    x = torch.empty((0, 2, 64), dtype=torch.bfloat16, device=DEV)
    dqt.dqt_rope_fwd(rope, [(x, x)])
    torch.cuda.synchronize()


def test_rope_leaves_what_lies_between(lib):
    """Rows of a wider buffer: what lies between them is not written, in place either."""
    log("rope: between rows")
    buf = torch.full((20, 3, 64 + 16), 7.0, dtype=torch.bfloat16, device=DEV)
    rope = dqt.rope(64, 32)
    dqt.dqt_rope_fwd(rope, [(buf[:, 1:3, :64], buf[:, 1:3, :64])])
    torch.cuda.synchronize()
    assert (buf[:, 0] == 7).all() and (buf[:, :, 64:] == 7).all() and (buf[:, 1:3, 32:64] == 7).all()
    assert not (buf[1:, 1:3, :32] == 7).any(-1).all()


def test_rope_gradient_by_differences(lib):
    """sum(g . rope(x)) moves by bwd(g) . dx: the map is linear, so a step of any size
    shows it to the fp32 roundings of the sums (64-bit here, 2^-24 of each term)."""
    log("rope: gradient against differences")
    gen = torch.Generator().manual_seed(7)
    rope = dqt.rope(64, 48, True, amp=1.3)
    x, g, dx = (torch.randn((11, 3, 64), generator=gen).to(DEV) for _ in range(3))
    pos = torch.randint(0, 9999, (11,), generator=gen, dtype=torch.int32).to(DEV)
    y = [torch.empty_like(x) for _ in range(3)]
    dqt.dqt_rope_fwd(rope, [(x, y[0]), ((x + dx), y[1])], pos)
    dqt.dqt_rope_bwd(rope, [(g, y[2])], pos)
    torch.cuda.synchronize()
    lhs = ((y[1].double() - y[0].double()) * g.double()).sum()
    rhs = (y[2].double() * dx.double()).sum()
    # each rotated value is off by 4 F32 (|a cos| + |b sin|) <= 6 F32 amp max(|a|, |b|); so is each gradient's
    bound = 16 * R.F32 * 1.3 * float(((x.abs() + dx.abs()) * 2 * g.abs().amax()).sum() + (g.abs() * 2 * dx.abs().amax()).sum())
    assert abs(float(lhs - rhs)) <= bound


def test_rope_non_finite_values_stay_in_their_pair(lib):
    log("rope: non-finite values")
    rope = dqt.rope(64, 64)
    x = torch.ones((5, 2, 64), device=DEV)
    x[2, 1, 3], x[3, 0, 40] = float("nan"), float("inf")
    y = torch.empty_like(x)
    dqt.dqt_rope_fwd(rope, [(x, y)])
    torch.cuda.synchronize()
    bad = ~torch.isfinite(y)
    want = torch.zeros_like(bad)
    want[2, 1, [3, 35]] = True
    want[3, 0, [8, 40]] = True
    assert torch.equal(bad, want)


def test_rope_other_stream_and_graph(lib):
    log("rope: captured and replayed on another stream")
    gen = torch.Generator().manual_seed(8)
    rope = dqt.rope(128)
    x = torch.randn((40, 4, 128), generator=gen).to(torch.bfloat16).to(DEV)
    pos = torch.arange(40, dtype=torch.int32, device=DEV)
    y, z = torch.empty_like(x), torch.empty_like(x)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    g = torch.cuda.CUDAGraph()
    with torch.cuda.stream(s):
        dqt.dqt_rope_fwd(rope, [(x, y)], pos)
        with torch.cuda.graph(g, stream=s):
            dqt.dqt_rope_fwd(rope, [(x, y)], pos)
    torch.cuda.current_stream().wait_stream(s)
    for k in range(4):
        pos.add_(1000 * k)
        g.replay()
        dqt.dqt_rope_fwd(rope, [(x, z)], pos)
        torch.cuda.synchronize()
        assert torch.equal(y, z)
