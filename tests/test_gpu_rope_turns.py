"""The sines and cosines of the rotation at angles where they lie next to a border of
fp32's rounding: the nearest fp32 value of the exact one, not its neighbour."""
import numpy as np
import pytest
import torch

from gpu_util import DEV, log
from paper_2412_04787_amd import dqt, model_step as MS

pytestmark = pytest.mark.gpu

TURN = 8 * np.arctan(np.longdouble(1))


def angles_beside_borders(rng, n, lo, hi, inverse, back):
    """n angles (64-bit fractions of a turn) whose sine (or cosine) lies 2^-47 to 2^-49 to either
    side of the middle between two fp32 values in lo .. hi, and the nearer of the two.  The fraction
    is off by 2^-65 of a turn; 64-bit mantissas by 2^-63."""
    f = rng.uniform(lo, hi, n).astype(np.float32)
    up = np.nextafter(f, np.float32(2))
    middle = (f.astype(np.longdouble) + up.astype(np.longdouble)) / 2
    side = rng.choice([-1, 1], n)
    value = middle + side * np.ldexp(np.longdouble(1), rng.integers(-49, -46, n))
    t = np.rint(inverse(value) / TURN * np.longdouble(2) ** 64).astype(np.uint64)
    assert (np.abs(back(t.astype(np.longdouble) / np.longdouble(2) ** 64 * TURN) - value) < 2.0 ** -60).all()
    return t, np.where(side < 0, f, up)


@pytest.mark.parametrize("quarter", [0, 1, 2, 3])
def test_turns_round_to_the_nearest(lib, quarter):
    """(1, 0) turned by t is (cos t, sin t).  A double's rounding is 2^-53 and the sums take some
    ten of them, each of what is below 1: less than 2^-49, so all round as the exact values do."""
    log(f"turns beside borders of fp32, quarter {quarter}")
    rng = np.random.default_rng(quarter)
    n = 512
    # both up to an eighth of a turn: sines up to 0.7071, cosines from there on
    s, want_s = angles_beside_borders(rng, n, 0.4, 0.7071, np.arcsin, np.sin)
    c, want_c = angles_beside_borders(rng, n, 0.7072, 0.9, np.arccos, np.cos)
    q = np.uint64(quarter) << np.uint64(62)
    for t, want, which in ((s, want_s, 1), (c, want_c, 0)):
        freq = torch.from_numpy((t + q).view(np.int64)).to(DEV)
        x = torch.zeros((1, 1, 1024), device=DEV)
        x[..., :512] = 1.0
        y = torch.empty_like(x)
        dqt.dqt_rope_fwd(dqt.Rope(freq, 1024), [(x, y)], torch.ones(1, dtype=torch.int32, device=DEV))
        torch.cuda.synchronize()
        got = y.cpu().numpy().reshape(2, 512)           # cos, sin
        # a quarter turn on: (cos, sin) -> (-sin, cos)
        for _ in range(quarter):
            got = np.stack((got[1], -got[0]))
        bad = got[which] != want
        assert not bad.any(), (int(bad.sum()), "sin" if which else "cos")


def test_the_model_keeps_one_form_of_its_angles(lib):
    """Frequencies with own_rope, tables of cosines and sines (2 tokens d bytes) without."""
    log("model: angles")
    for name, own in (("tiny_rope", True), ("tiny_ops", False)):
        m = MS.DQTModel(MS.MODELS[name])
        assert hasattr(m, "rope") == own and hasattr(m, "cos") != own and hasattr(m, "sin") != own
