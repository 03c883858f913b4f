"""Attention over the 8-bit cache where a block has more pages than it looks up at a
time, rows have more parts than are joined at a time, and caches are read past the
last-level one: against float64, with the kernel that runs and the number of parts checked,
so that another choice of tile or parts does not leave a path without a test.

Contexts are long, caches small: a sequence's row of the table names the same pages
again and again."""
import warnings

import numpy as np
import pytest
import torch

import kv_reference as R
from gpu_util import DEV, log
from paper_2412_04787_amd import dqt
from test_gpu_kv import FILL, SENT, dev32, device_cache, random_cache

pytestmark = pytest.mark.gpu


def launched(call):
    """Names of the library's kernels that a call launches (none where nothing can be traced)."""
    from torch.profiler import ProfilerActivity, profile
    torch.cuda.synchronize()
    with warnings.catch_warnings():
        warnings.simplefilter("ignore")
        with profile(activities=[ProfilerActivity.CUDA]) as p:
            call()
            torch.cuda.synchronize()
        return [e.name for e in p.events() if "dqt::" in e.name]


def values(h, fmt, row, n):
    """float64 keys and values [n, kvh, d] of a sequence's first n tokens, and which of them lie in a page."""
    p = torch.as_tensor(np.asarray(row[:-(-n // R.PAGE)], dtype=np.int64), device=DEV)
    there = (p >= 0) & (p < h.K.shape[0])
    p = p.clamp(0, h.K.shape[0] - 1)
    k, v = (x.view(torch.uint8)[p].view(R.DTYPE[fmt]).float().double() * h.scales[p, :, j].double()[..., None, None]
            for j, x in enumerate((h.K, h.V)))
    kvh, d = h.K.shape[1], h.K.shape[3]
    return (k.permute(0, 2, 1, 3).reshape(-1, kvh, d)[:n], v.permute(0, 3, 1, 2).reshape(-1, kvh, d)[:n],
            there.repeat_interleave(R.PAGE)[:n])


def check(fmt, d, heads, kvh, lq, lk, kernel, parts, width=None, none=False, causal=True, holes=(), seed=0):
    """kernel: the name of the attention's kernel; parts: a test of the number that rows may have."""
    rng, gen = np.random.default_rng(seed), torch.Generator().manual_seed(seed)
    held, n = [-(-x // R.PAGE) for x in lk], len(lk)
    common = 60
    c = random_cache(gen, common + n, kvh, d, fmt)
    table = np.full((n, max(held + [1]) if width is None else width), -1, np.int32)
    for i, x in enumerate(held):
        table[i, :x] = rng.integers(0, common, x)
        if lk[i] % R.PAGE:                            # (the last page is the sequence's own: NaN behind its end)
            table[i, x - 1] = common + i
            c.K[common + i, :, lk[i] % R.PAGE:] = FILL[fmt]
            c.V[common + i, :, :, lk[i] % R.PAGE:] = FILL[fmt]
    for i, p, x in holes:
        table[i, p] = x
    h, tq = device_cache(c), sum(lq)
    Q = torch.randn((tq, heads, d), generator=gen).to(torch.bfloat16).to(DEV)
    O, lse = torch.full((tq, heads, d), SENT, dtype=torch.bfloat16, device=DEV), torch.full((heads, tq), SENT, device=DEV)
    qs = np.concatenate([[0], np.cumsum(lq)])
    b = dqt.kv_batch(dev32(table), dev32(lk), tq, heads, None if none else dev32(qs), causal=causal)
    need = dqt.dqt_kv_attn_workspace(h, b)
    ws = dqt.workspace(need)
    if ws is not None:
        ws.fill_(float("nan"))
    names = launched(lambda: dqt.dqt_kv_attn(h, b, Q, O, lse, ws))
    most = max(1, need // (tq * heads * (d + 1) * 4))
    log(f"  {most} parts, {names}")
    assert parts(most), most
    assert not names or any(kernel in x for x in names), names
    for i in range(n):
        a, z = int(qs[i]), int(qs[i + 1])
        K, V, there = values(h, fmt, table[i], lk[i])
        for j in range(kvh):
            hs = slice(j * (heads // kvh), (j + 1) * (heads // kvh))
            with torch.device(DEV):
                r = R.attention(Q[a:z, hs], K[:, j:j + 1], V[:, j:j + 1], there, d ** -0.5, causal)
            for name, g, ref, t in (("O", O[a:z, hs].double(), r["O"], r["t_O"]), ("lse", lse[hs, a:z].double(), r["lse"], r["t_lse"])):
                bad = ~((g - ref).abs() <= t + 1e-30) & ~((g == ref) & torch.isinf(ref))
                assert not bad.any(), (name, i, j, int(bad.sum()), bad.nonzero()[0].tolist(), float((g - ref).abs().max()))
    return names


one = lambda p: p == 1
flag = lambda fmt: "true" if fmt == "e4m3" else "false"


@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
@pytest.mark.parametrize("d", [64, 128])
def test_many_rows_more_pages_than_a_window(lib, fmt, d):
    """Tiles of 128 rows, unsplit, over more than 128 pages: an odd number of them, ends and
    holes in the second window and at its border, with the mask and without."""
    log(f"chunks over more than 128 pages {fmt} d={d}")
    kernel = f"kv_tile_kernel<{d}, {flag(fmt)}>"
    check(fmt, d, 86, 2, [380], [8361], kernel, one, holes=[(0, 129, -1)], seed=1)
    check(fmt, d, 86, 2, [190, 190], [12345, 8257], kernel, one, holes=[(0, 127, -1), (0, 128, 1 << 20), (0, 130, -1)], seed=2)
    check(fmt, d, 86, 2, [380], [8193], kernel, one, causal=False, holes=[(0, 0, -1)], seed=3)


@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
@pytest.mark.parametrize("heads", [2, 20])            # tiles of 16 and of 32 rows
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("past", [False, True])       # past the last-level cache or not
def test_few_rows_more_pages_than_a_window(lib, fmt, d, heads, past):
    """Rows over more than 256 pages to a block, by as many tokens as 32 parts of 256 pages do
    not hold; a cache of more than 256 MB (as far as the table says) is read past the last level."""
    log(f"single tokens over more than 256 pages to a block {fmt} d={d} heads={heads} past={past}")
    width = (1 << 28) // (2 * d * 64) + 100 if past else 9376
    kernel = f"kv_attn_kernel<{d}, {flag(fmt)}, {1 if heads == 2 else 2}, {'true' if past else 'false'}>"
    chunk = -(-width // 32)
    assert chunk > 256
    check(fmt, d, heads, 1, [1], [300001], kernel, lambda p: 1 < p <= 32 and width // p > 256, width=width, none=True,
          holes=[(0, 3, -1), (0, 258, -1), (0, 4600, 1 << 25)], seed=4)


@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
@pytest.mark.parametrize("heads", [4, 40])
@pytest.mark.parametrize("d", [64, 128])
def test_short_sequences_of_a_large_cache(lib, fmt, heads, d):
    """Ordinary lengths, none and one among them, in a batch whose cache is read past the last
    level; whole and in parts."""
    log(f"short sequences of a large cache {fmt} d={d} heads={heads}")
    kernel = f"kv_attn_kernel<{d}, {flag(fmt)}, {1 if heads == 4 else 2}, true>"
    for n, seed in ((5, 5), (300, 6)):
        lk = [1, 0, 64, 1000, 20001] if n == 5 else np.random.default_rng(7).integers(0, 200, n).tolist()
        check(fmt, d, heads, 2, [1] * n, lk, kernel, lambda p: p >= 1, width=(1 << 28) // (2 * 2 * d * 64 * n) + 10, none=True, seed=seed)


@pytest.mark.parametrize("fmt,d,heads,kvh", [("int8", 64, 32, 16), ("e4m3", 64, 32, 4), ("e4m3", 128, 32, 16), ("int8", 128, 33, 33)])
def test_joined_rows_of_more_parts_than_a_round(lib, fmt, d, heads, kvh):
    """More than 4096 rows of more than 16 parts: heads that are no multiple of 4 too."""
    log(f"many rows of many parts {fmt} d={d} heads={heads}/{kvh}")
    names = check(fmt, d, heads, kvh, [129], [131072], "kv_", lambda p: p > 16, holes=[(0, 5, -1), (0, 2000, -1)], seed=8)
    assert not names or any(f"kv_join_heads_kernel<{d}>" in x for x in names)
