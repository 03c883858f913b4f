"""The 8-bit cache of keys and values: dqt_kv_append, dqt_kv_attn and dqt_kv_copy
against plain implementations, page by page and in 64 bits; the calls together, as
decoding makes them."""
import numpy as np
import pytest
import torch

import kv_reference as R
from gpu_util import DEV, log
from paper_2412_04787_amd import dqt

pytestmark = pytest.mark.gpu

SENT = 1.25e4
FMT = {"e4m3": dqt.DQT_FP8E4M3, "int8": dqt.DQT_I8}
FILL = {"e4m3": 0x7F, "int8": 0x80}        # a NaN; -128, which is never written


def device_cache(c):
    """The library's handle of a copy of a CPU cache."""
    dt = R.DTYPE[c.fmt]
    return dqt.KvCache(c.K.to(DEV).view(dt), c.V.to(DEV).view(dt), c.scales.to(DEV))


def same_cache(h, c, pages=slice(None)):
    for name, a, b in (("scales", h.scales, c.scales), ("K", h.K.view(torch.uint8), c.K), ("V", h.V.view(torch.uint8), c.V)):
        a = a.cpu()[pages]
        assert torch.equal(a, b[pages]), (name, (a != b[pages]).nonzero()[:4].tolist())


def dev32(x):
    return torch.from_numpy(np.ascontiguousarray(x, dtype=np.int32)).to(DEV)


def page_table(rng, lens, spare=3, extra=0):
    """A table of shuffled pages for sequences of those lengths, and the pages in all."""
    held = [-(-n // R.PAGE) for n in lens]
    pages = sum(held) + spare
    order, at = rng.permutation(pages), 0
    table = np.full((len(lens), max(held + [1]) + extra), -1, np.int32)
    for i, n in enumerate(held):
        table[i, :n] = order[at:at + n]
        at += n
    return table, pages


def strided(x, layout):
    """A device view of x [tokens, heads, d]."""
    if layout == "heads":
        return x.permute(1, 0, 2).contiguous().to(DEV).permute(1, 0, 2)
    if layout == "wide":
        buf = torch.full((x.shape[0], 2, x.shape[1] + 1, x.shape[2] + 8), 7.0, dtype=x.dtype)
        buf[:, 1, :x.shape[1], :x.shape[2]] = x
        return buf.to(DEV)[:, 1, :x.shape[1], :x.shape[2]]
    return x.to(DEV)


def starts(lq, before=0):
    return np.concatenate([[0], np.cumsum(lq)]) + before


# ------------------------------------------------------------------ append

@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
@pytest.mark.parametrize("d,kvh", [(64, 1), (128, 3)])
def test_append_in_pieces(lib, fmt, d, kvh):
    """Sequences grow by pieces of different lengths, single tokens among them, values
    of growing size (the scale rises within a page); every byte of the cache, written
    or not, is the plain implementation's.  Without rotation each code is exact."""
    log(f"append in pieces {fmt} d={d} kv_heads={kvh}")
    rng, gen = np.random.default_rng(d), torch.Generator().manual_seed(d + kvh)
    total = [333, 64, 1, 0, 130]
    table, pages = page_table(rng, total, extra=1)
    c = R.Cache(pages, kvh, d, fmt, FILL[fmt])
    h, have = device_cache(c), [0] * len(total)
    kv_len, tab = torch.zeros(len(total), dtype=torch.int32, device=DEV), dev32(table)
    for piece in (1, 5, 1, 1, 60, 64, 65, 1, 127, 2, 1):
        lq = [min(piece, n - m) for n, m in zip(total, have)]
        tq = sum(lq)
        K, V = (torch.randn((tq, kvh, d), generator=gen) * torch.exp(torch.rand((tq, 1, 1), generator=gen) * 6 - 4) for _ in range(2))
        K, V = K.to(torch.bfloat16), V.to(torch.bfloat16)
        have = [m + q for m, q in zip(have, lq)]
        kv_len.copy_(dev32(have))
        b = dqt.kv_batch(tab, kv_len, tq, kvh, dev32(starts(lq)))
        dqt.dqt_kv_append(h, b, K.to(DEV), V.to(DEV))
        at = 0
        for i, q in enumerate(lq):
            c.write(table[i], have[i] - q, K[at:at + q].float(), V[at:at + q].float())
            at += q
        torch.cuda.synchronize()
        same_cache(h, c)


@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
def test_append_single_tokens(lib, fmt):
    """One token for each sequence without starts, as decoding calls it; a token again
    at the same place, and a page begun anew after its sequence ended."""
    log(f"append single tokens {fmt}")
    rng, gen = np.random.default_rng(1), torch.Generator().manual_seed(1)
    lens = np.array([1, 64, 65, 17, 128, 2, 0, 63])
    table, pages = page_table(rng, lens + 3)
    c = R.Cache(pages, 2, 64, fmt, 5)
    c.scales.fill_(4.0)                    # (scales that stand are powers of two)
    h, tab = device_cache(c), dev32(table)
    for step in range(5):
        at = lens + (0, 1, 1, 2, -1)[step]
        K, V = ((torch.randn((8, 2, 64), generator=gen) * (1 + 9 * (step == 1))).to(torch.bfloat16) for _ in range(2))
        dqt.dqt_kv_append(h, dqt.kv_batch(tab, dev32(at), 8, 2), K.to(DEV), V.to(DEV))
        for i in range(8):
            if at[i] > 0:
                c.write(table[i], at[i] - 1, K[i:i + 1].float(), V[i:i + 1].float())
        torch.cuda.synchronize()
        same_cache(h, c)


@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
def test_append_values_of_all_sizes(lib, fmt):
    """Zeros, the border of a scale, the smallest and largest scales, infinities and NaN."""
    log(f"append: values of all sizes {fmt}")
    top = R.TOP[fmt]
    inf, nan = float("inf"), float("nan")
    rows = [[0.0], [top], [top * 1.01], [top * 2.0 ** -3, -1.0], [2.0 ** -70, -(2.0 ** -74)], [3e38], [inf, 1.0], [-inf, nan, 0.5],
            [nan], [2.0 ** -133], [top * 2.0 ** 112, -1e30], [1.0, -0.0, 2.0 ** -12, 0.4375, 0.40625]]
    n = len(rows)
    x = torch.zeros((n, 1, 64))
    for i, r in enumerate(rows):
        x[i, 0, 5:5 + len(r)] = torch.tensor(r)
    x = x.to(torch.bfloat16)
    table = np.arange(n, dtype=np.int32)[:, None]
    c = R.Cache(n, 1, 64, fmt, 0)
    h = device_cache(c)
    dqt.dqt_kv_append(h, dqt.kv_batch(dev32(table), dev32([1] * n), n, 1), x.to(DEV), x.to(DEV))
    for i in range(n):
        c.write(table[i], 0, x[i:i + 1].float(), x[i:i + 1].float())
    torch.cuda.synchronize()
    same_cache(h, c)


@pytest.mark.parametrize("layout", ["plain", "heads", "wide"])
@pytest.mark.parametrize("pairs", [False, True])
@pytest.mark.parametrize("d,rot", [(64, 64), (128, 48), (128, 128)])
def test_append_rotates(lib, layout, pairs, d, rot):
    """Keys are rotated before they are written, queries beside them; positions follow
    from the lengths.  A code is within half a step of the exact value (and the fp32
    roundings of the rotation)."""
    log(f"append rotates d={d} rot={rot} pairs={pairs} {layout}")
    rng, gen = np.random.default_rng(2), torch.Generator().manual_seed(d + rot)
    heads, kvh, before, behind = 6, 2, 3, 4
    lq, lk = [70, 1, 0, 33, 129], [70, 200, 9, 97, 1000]
    table, pages = page_table(rng, lk)
    tq = sum(lq) + before + behind
    Q, K, V = (torch.randn((tq, n, d), generator=gen).to(torch.bfloat16) for n in (heads, kvh, kvh))
    freqs = dict(factor=8.0, context=256.0)
    f = dqt.dqt_rope_freqs(rot, **freqs)
    rope = dqt.rope(d, rot, pairs, 1.2079, **freqs)
    for fmt in ("e4m3", "int8"):
        c = R.Cache(pages, kvh, d, fmt, 0)
        c.scales.fill_(2.0 ** -20)         # (what stands in the page is on a small scale)
        h = device_cache(c)
        Qd = strided(Q, layout)
        Qr = torch.full((tq, heads, d), SENT, dtype=torch.bfloat16, device=DEV)
        b = dqt.kv_batch(dev32(table), dev32(lk), tq, heads, dev32(starts(lq, before)))
        dqt.dqt_kv_append(h, b, strided(K, layout), strided(V, layout), rope, Qd, Qr)
        dqt.dqt_kv_append(h, b, strided(K, layout), strided(V, layout), rope, Qd, Qd)      # again, queries in place
        torch.cuda.synchronize()
        assert (Qr[:before] == SENT).all() and (Qr[tq - behind:] == SENT).all()
        assert torch.equal(Qd[before:tq - behind], Qr[before:tq - behind])
        got = R.Cache(pages, kvh, d, fmt, 0)
        got.K, got.V, got.scales = h.K.view(torch.uint8).cpu(), h.V.view(torch.uint8).cpu(), h.scales.cpu()
        at = before
        for i, (q, n) in enumerate(zip(lq, lk)):
            pos, rows = np.arange(n - q, n), slice(at, at + q)
            at += q
            if q == 0:
                continue
            y, t = R.rotate(Q[rows], pos, f, rot, pairs, 1.2079)
            err = (Qr[rows].double().cpu() - y).abs()
            assert (err <= t + R.BF16 * y.abs() * (1 + R.BF16)).all()
            y, t = R.rotate(K[rows], pos, f, rot, pairs, 1.2079)
            kk, vv, _ = got.values(table[i], n, pages)
            kk, vv = kk[n - q:], vv[n - q:]
            page = torch.as_tensor(table[i][pos // R.PAGE].astype(np.int64))
            for x, have, slack, j in ((y, kk, t, 0), (V[rows].double(), vv, torch.zeros_like(y), 1)):
                s = got.scales[page, :, j].double()[..., None]
                step = 0.5 * s if fmt == "int8" else torch.maximum(x.abs() * 2.0 ** -4, s * 2.0 ** -10)
                assert ((have - x).abs() <= step + 2 * slack + 1e-30).all()
                # the scale: of the page's largest value
                for p in np.unique(pos // R.PAGE):
                    m = x[torch.as_tensor(pos // R.PAGE == p)].abs().amax((0, 2))
                    sc = got.scales[int(table[i][p]), :, j].double()
                    top = R.TOP[fmt]
                    assert (m <= top * sc * (1 + 1e-6)).all() and (m * (1 + 1e-6) > top * sc / 2).all()


def test_append_outside(lib):
    """Pages outside the cache, more new tokens than the length holds, lengths past
    max_len: nothing but the tokens that have a place is written."""
    log("append: outside")
    gen = torch.Generator().manual_seed(3)
    c = R.Cache(4, 1, 64, "e4m3", 9)
    c.scales.fill_(0.5)
    h = device_cache(c)
    table = np.array([[0, -1], [9, 1], [2, 7], [3, 3]], np.int32)
    lq, lk = [70, 70, 8, 3], [70, 70, 5, 500]
    K, V = (torch.randn((sum(lq), 1, 64), generator=gen).to(torch.bfloat16) for _ in range(2))
    rope = dqt.rope(64)
    f = dqt.dqt_rope_freqs(64)
    Qr = torch.full((sum(lq), 1, 64), SENT, dtype=torch.bfloat16, device=DEV)
    dqt.dqt_kv_append(h, dqt.kv_batch(dev32(table), dev32(lk), sum(lq), 1, dev32(starts(lq)), max_len=70), K.to(DEV), V.to(DEV))
    c.write(table[0], 0, K[:70].float(), V[:70].float())
    c.write(table[1], 0, K[70:140].float(), V[70:140].float())
    c.write(table[2], 0, K[143:148].float(), V[143:148].float())
    c.write(table[3], 67, K[148:].float(), V[148:].float())
    torch.cuda.synchronize()
    same_cache(h, c)
    dqt.dqt_kv_append(h, dqt.kv_batch(dev32(table), dev32(lk), sum(lq), 1, dev32(starts(lq)), max_len=70), K.to(DEV), V.to(DEV),
                      rope, K.to(DEV), Qr)
    torch.cuda.synchronize()
    y, t = R.rotate(K[140:148], np.arange(-3, 5), f, 64, False)
    assert (Qr[140:143] == SENT).all()
    assert ((Qr[143:148].double().cpu() - y[3:]).abs() <= (t + R.BF16 * y.abs() * 1.01)[3:]).all()
    y, t = R.rotate(K[70:140], np.arange(70), f, 64, False)
    assert ((Qr[70:140].double().cpu() - y).abs() <= t + R.BF16 * y.abs() * 1.01).all()


# ------------------------------------------------------------------ attention

def random_cache(gen, pages, kvh, d, fmt, std=1.0):
    """Codes of random tokens, scales that differ from page to page and head to head."""
    c = R.Cache(pages, kvh, d, fmt, 0)
    for buf in (c.K, c.V):
        x = torch.randn(buf.shape, generator=gen) * (R.TOP[fmt] / 5)
        buf.copy_(R.encode(x, fmt))
    e = torch.randint(-2, 2, c.scales.shape, generator=gen).float()
    c.scales = torch.exp2(e - (7 if fmt == "e4m3" else 5)) * std
    return c


def run_attn(fmt, d, heads, kvh, lq, lk, causal=True, layout="plain", scale=None, seed=0, before=0, behind=0, max_len=None,
             none=False, holes=(), std=1.0, qstd=1.0, extra=0):
    rng, gen = np.random.default_rng(seed), torch.Generator().manual_seed(seed)
    table, pages = page_table(rng, lk, extra=extra)
    c = random_cache(gen, pages, kvh, d, fmt, std)
    for i, n in enumerate(lk):                       # behind a sequence's end: NaN, or codes that are never written
        if n % R.PAGE:
            c.K[table[i, n // R.PAGE], :, n % R.PAGE:] = FILL[fmt]
            c.V[table[i, n // R.PAGE], :, :, n % R.PAGE:] = FILL[fmt]
    for i, p, x in holes:
        table[i, p] = x
    tq = sum(lq) + before + behind
    Q = (torch.randn((tq, heads, d), generator=gen) * qstd).to(torch.bfloat16)
    Qd = strided(Q, layout)
    O = torch.full((tq, heads, d), SENT, dtype=torch.bfloat16)
    O = strided(O, layout)
    lse = torch.full((heads, tq), SENT, device=DEV)
    h = device_cache(c)
    qs = starts(lq, before)
    b = dqt.kv_batch(dev32(table), dev32(lk), tq, heads, None if none else dev32(qs), max_len, scale, causal)
    ws = dqt.workspace(dqt.dqt_kv_attn_workspace(h, b))
    if ws is not None:
        ws.fill_(float("nan"))
    dqt.dqt_kv_attn(h, b, Qd, O, lse, ws)
    torch.cuda.synchronize()
    got, gl = O.double().cpu(), lse.double().cpu()
    own = torch.zeros(tq, dtype=torch.bool)
    for i, n in enumerate(lk):
        a, z = int(qs[i]), int(qs[i + 1])
        own[a:z] = True
        K, V, there = c.values(table[i], n, pages)
        r = R.attention(Q[a:z], K, V, there, d ** -0.5 if scale is None else scale, causal)
        for name, g, ref, t in (("O", got[a:z], r["O"], r["t_O"]), ("lse", gl[:, a:z], r["lse"], r["t_lse"])):
            bad = ~((g - ref).abs() <= t + 1e-30) & ~((g == ref) & torch.isinf(ref))
            assert not bad.any(), (name, i, int(bad.sum()), bad.nonzero()[0].tolist(), float((g - ref).abs().max()))
    assert (O.cpu()[~own] == SENT).all() and (gl[:, ~own] == SENT).all()


LENGTHS = [
    # (new tokens, lengths)
    ([1], [1]),
    ([1], [64]),
    ([37], [37]),
    ([1, 1, 1, 1, 1, 1, 1], [1, 2, 63, 64, 65, 130, 1000]),
    ([3, 1, 5, 2], [70, 500, 131, 129]),
    ([64, 65, 1, 63], [64, 65, 1, 63]),
    ([40, 3, 200, 130], [100, 500, 231, 700]),
    ([9, 10, 0, 0], [4, 0, 30, 0]),                  # rows that see nothing; no tokens; no queries
]


@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("li", range(len(LENGTHS)))
@pytest.mark.parametrize("heads,kvh", [(2, 2), (6, 2), (8, 1)])
def test_attention_matches_float64(lib, fmt, d, li, heads, kvh):
    lq, lk = LENGTHS[li]
    log(f"cache attention {fmt} d={d} heads={heads}/{kvh} lq={lq} lk={lk}")
    run_attn(fmt, d, heads, kvh, lq, lk, seed=li)


@pytest.mark.parametrize("d", [64, 128])
def test_attention_groups(lib, d):
    """Group sizes from 1 to more rows than a tile of few rows has."""
    log(f"cache attention: groups d={d}")
    for g in (1, 3, 5, 16, 17, 24, 40):
        run_attn("e4m3", d, 2 * g, 2, [1, 1, 1], [70, 1, 333], seed=g, none=True)
    run_attn("int8", d, 33, 1, [2, 1, 7], [70, 1, 333], seed=41)


@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
@pytest.mark.parametrize("d", [64, 128])
def test_attention_without_mask(lib, fmt, d):
    log(f"cache attention not causal {fmt} d={d}")
    run_attn(fmt, d, 4, 2, [1, 70, 129, 0], [200, 3, 129, 5], causal=False, seed=20)


@pytest.mark.parametrize("layout", ["heads", "wide"])
def test_attention_strides(lib, layout):
    log(f"cache attention strides {layout}")
    run_attn("e4m3", 64, 6, 3, [33, 100, 1], [90, 100, 300], layout=layout, seed=21)
    run_attn("int8", 128, 6, 3, [2, 1, 1], [90, 100, 1300], layout=layout, seed=21)


def test_attention_leaves_other_tokens(lib):
    log("cache attention: tokens before the first and behind the last sequence")
    run_attn("e4m3", 128, 4, 2, [20, 75], [20, 80], before=13, behind=29, seed=22)
    run_attn("int8", 64, 4, 4, [1, 1], [2100, 20], before=3, behind=5, seed=23)


def test_attention_many_sequences(lib):
    rng = np.random.default_rng(3)
    lq = rng.integers(0, 9, 200).tolist()
    lk = [x + int(c) for x, c in zip(lq, rng.integers(0, 90, 200))]
    log("cache attention: 200 sequences")
    run_attn("e4m3", 64, 3, 1, lq, lk, seed=24)
    run_attn("int8", 128, 2, 2, [1] * 130, rng.integers(1, 140, 130).tolist(), seed=25, none=True)


def test_attention_many_sequences_of_many_rows(lib):
    """More sequences than lanes, each with more rows than a tile of few rows: chunks,
    and single tokens of large groups without starts."""
    rng = np.random.default_rng(4)
    lq = rng.integers(0, 70, 90).tolist()
    lk = [x + int(c) for x, c in zip(lq, rng.integers(0, 150, 90))]
    log("cache attention: 90 sequences of chunks, 70 of groups of 200")
    run_attn("int8", 64, 2, 1, lq, lk, seed=42)
    run_attn("e4m3", 64, 200, 1, [1] * 70, rng.integers(0, 140, 70).tolist(), seed=43, none=True)
    run_attn("e4m3", 128, 260, 2, [1, 1], [300, 70], seed=44, none=True)


def test_thousands_of_sequences(lib):
    """3000 sequences of one new token: every page is the plain implementation's, every
    row that of its sequence."""
    log("append and attention: 3000 sequences")
    rng, gen = np.random.default_rng(6), torch.Generator().manual_seed(6)
    n = 3000
    lens = rng.integers(0, 70, n)
    table, pages = page_table(rng, lens.tolist())
    c = random_cache(gen, pages, 1, 64, "e4m3")
    h = device_cache(c)
    K, V, Q = (torch.randn((n, x, 64), generator=gen).to(torch.bfloat16) for x in (1, 1, 2))
    b = dqt.kv_batch(dev32(table), dev32(lens), n, 2)
    O = torch.full((n, 2, 64), SENT, dtype=torch.bfloat16, device=DEV)
    dqt.dqt_kv_append(h, b, K.to(DEV), V.to(DEV))
    dqt.dqt_kv_attn(h, b, Q.to(DEV), O, None, dqt.workspace(dqt.dqt_kv_attn_workspace(h, b)))
    torch.cuda.synchronize()
    for i in range(n):
        if lens[i]:
            c.write(table[i], lens[i] - 1, K[i:i + 1].float(), V[i:i + 1].float())
    same_cache(h, c)
    got = O.double().cpu()
    for i in range(0, n, 7):
        k, v, there = c.values(table[i], int(lens[i]), pages)
        r = R.attention(Q[i:i + 1], k, v, there, 0.125, True)
        assert ((got[i:i + 1] - r["O"]).abs() <= r["t_O"]).all(), (i, int(lens[i]))


def test_starts_and_lengths_out_of_range(lib):
    """Values that break the rules are clamped: sequences that follow them are right, and
    tokens outside every sequence stay as they are."""
    log("append and attention: starts and lengths out of range")
    gen = torch.Generator().manual_seed(9)
    c = random_cache(gen, 6, 1, 64, "int8")
    table = np.arange(6, dtype=np.int32).reshape(3, 2)
    for heads in (1, 64):                             # tiles of few rows, and of many
        for qs, lk, good in (([-7, 3, 5, 9], [50, 90, 1 << 30], {0: (0, 3, 50), 1: (3, 5, 90), 2: (5, 9, 128)}),
                             ([0, 1 << 30, 4, 6], [-5, 100, 64], {2: (4, 6, 64)}),
                             ([9, 9, 2, 2 ** 31 - 1], [3, 100, 128], {2: (2, 9, 128)})):
            h = device_cache(c)
            Q = torch.randn((9, heads, 64), generator=gen).to(torch.bfloat16)
            O = torch.full((9, heads, 64), SENT, dtype=torch.bfloat16, device=DEV)
            b = dqt.kv_batch(dev32(table), dev32(lk), 9, heads, dev32(qs))
            dqt.dqt_kv_attn(h, b, Q.to(DEV), O, None, dqt.workspace(dqt.dqt_kv_attn_workspace(h, b)))
            torch.cuda.synchronize()
            for s, (x, y, n) in good.items():
                k, v, there = c.values(table[s], n, 6)
                r = R.attention(Q[x:y], k, v, there, 0.125, True)
                assert ((O[x:y].double().cpu() - r["O"]).abs() <= r["t_O"]).all(), (heads, qs, s)
            kv = torch.randn((9, 1, 64), generator=gen).to(torch.bfloat16).to(DEV)
            dqt.dqt_kv_append(h, dqt.kv_batch(dev32(table), dev32(lk), 9, 1, dev32(qs)), kv, kv)
            torch.cuda.synchronize()


@pytest.mark.parametrize("rows", [1, 3, 40])
def test_no_table(lib, rows):
    """max_len = 0 needs no table, whatever table_stride says: nothing is seen, nothing is written."""
    n, heads, kvh, d = 3, 8, 2, 64
    h = dqt.kv_cache(2, kvh, d, FMT["e4m3"], device=DEV)
    h.K.view(torch.uint8).fill_(3)
    h.scales.fill_(1.0)
    x = torch.randn(n * rows, heads, d, dtype=torch.bfloat16, device=DEV)
    kv_len, q_start = dev32([0, rows, 9]), dev32(starts([rows] * n))
    desc = dqt.DqtKvBatch(None, kv_len.data_ptr(), None if rows == 1 else q_start.data_ptr(), n * rows, 0, n, 1 << 20, heads, 1,
                          0.125, 0)
    batch = dqt.KvBatch(desc, (kv_len, q_start), 0.125)
    o, lse = torch.full_like(x, SENT), torch.full((heads, n * rows), SENT, device=DEV)
    dqt.dqt_kv_append(h, batch, x[:, :kvh], x[:, :kvh])
    assert dqt.dqt_kv_attn_workspace(h, batch) == 0
    dqt.dqt_kv_attn(h, batch, x, o, lse)
    torch.cuda.synchronize()
    assert (o == 0).all() and (lse == -float("inf")).all()
    assert (h.K.view(torch.uint8) == 3).all() and (h.scales == 1.0).all()


def test_attention_long(lib):
    log("cache attention: one token over 20001, five over 9000, a chunk over 5000; room for more than there is")
    run_attn("e4m3", 128, 4, 1, [1], [20001], seed=27)
    run_attn("int8", 64, 2, 2, [1, 5], [77, 9000], seed=28, extra=300)
    run_attn("e4m3", 64, 4, 2, [129, 300], [5000, 300], seed=29, extra=40)
    run_attn("int8", 128, 2, 1, [150], [3000], seed=30, max_len=3001)


@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
@pytest.mark.parametrize("d", [64, 128])
def test_attention_chunks_of_many_heads(lib, fmt, d):
    """As many tiles of 128 rows as there are compute units, or a few less: one sequence,
    three of odd lengths with holes and rows that see nothing, strided."""
    log(f"cache attention: chunks of 85 heads {fmt} d={d}")
    run_attn(fmt, d, 85, 85, [384], [384], seed=50)
    run_attn(fmt, d, 85, 85, [127, 100, 128], [127, 60, 301], seed=51, holes=[(2, 1, -1), (2, 4, 1 << 20)], layout="wide")
    run_attn(fmt, d, 170, 85, [60, 64, 0, 57], [64, 65, 9, 70], causal=False, seed=52, before=5, behind=3)


@pytest.mark.parametrize("fmt,d", [("e4m3", 128), ("int8", 128)])
def test_attention_long_chunk(lib, fmt, d):
    """Tiles of 128 rows whose pages are split, and those of fewer rows."""
    log(f"cache attention: a chunk over 5000 tokens {fmt} d={d}")
    run_attn(fmt, d, 42, 42, [384], [5000], seed=53)
    run_attn(fmt, d, 8, 4, [200, 90], [5000, 2100], seed=54, holes=[(0, 7, -1)])


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("heads,kvh", [(40, 8), (39, 13), (10, 5), (5, 5), (9, 9)])
def test_attention_joined_rows(lib, d, heads, kvh):
    """More than 4096 rows of several parts: numbers of heads that are no multiple of 4,
    rows of one part and of none beside them, tokens of no sequence."""
    log(f"cache attention: joined rows d={d} heads={heads}/{kvh}")
    n, far = 4200 // heads + 2, 3000 if d == 128 else 9000
    run_attn("e4m3", d, heads, kvh, [n - 9, 7, 3], [far, 2, far - 500], seed=55, before=2, behind=6)
    run_attn("int8", d, heads, kvh, [n], [far - 700], seed=56, causal=False, holes=[(0, i, -1) for i in range(4, 30)])


@pytest.mark.parametrize("d", [64, 128])
def test_attention_joined_single_tokens(lib, d):
    """Thousands of rows of several parts, one token a sequence."""
    log(f"cache attention: joined rows of single tokens d={d}")
    lk = [1, 0, 3000, 1500, 700, 64, 65, 4100 if d == 128 else 9000, 2000]
    run_attn("e4m3", d, 512, 4, [1] * 9, lk, seed=57, none=True)
    run_attn("int8", d, 250, 2, [1] * 17, lk + [1000] * 8, seed=58)


def test_attention_holes(lib):
    """Pages outside the cache hold no tokens: at the start, the end, all of them."""
    log("cache attention: holes")
    run_attn("e4m3", 64, 4, 2, [1, 3, 80, 2], [300, 200, 400, 70], seed=31,
             holes=[(0, 0, -1), (0, 4, 1 << 30), (1, 3, -5), (2, 1, 99999), (2, 2, -1), (3, 0, -1), (3, 1, -1)])
    run_attn("int8", 128, 8, 1, [1, 1], [1500, 64], seed=32, holes=[(0, i, -1) for i in range(3, 20)] + [(1, 0, -2)])


def test_attention_scales_and_large_scores(lib):
    """Scores of hundreds; tiny and large scales; queries far from one."""
    log("cache attention: large scores, scales")
    run_attn("e4m3", 64, 4, 2, [1, 40], [300, 300], scale=2.0, seed=33)
    run_attn("int8", 128, 2, 1, [3], [700], scale=0.5, seed=34)
    run_attn("e4m3", 64, 2, 1, [1, 70], [500, 200], seed=35, std=2.0 ** 30, qstd=2.0 ** -30)
    run_attn("int8", 64, 2, 1, [1, 70], [500, 200], seed=36, std=2.0 ** -30, qstd=2.0 ** 30)
    run_attn("e4m3", 128, 2, 1, [1, 70], [500, 200], seed=37, qstd=1e-30)


def test_attention_value_scales_apart(lib):
    """Values whose pages differ by 2^40, the large ones first, last and alone."""
    log("cache attention: pages of very different values")
    gen = torch.Generator().manual_seed(5)
    for big in ([0], [3], [1, 2], []):
        c = random_cache(gen, 4, 1, 64, "e4m3")
        for p in big:
            c.scales[p, :, 1] *= 2.0 ** 40
        if not big:
            c.V[1] = 0
            c.scales[1, :, 1] = 2.0 ** -64
        table = np.array([[0, 1, 2, 3]], np.int32)
        h = device_cache(c)
        for n in (1, 40):
            Q = torch.randn((n, 2, 64), generator=gen).to(torch.bfloat16)
            O = torch.empty((n, 2, 64), dtype=torch.bfloat16, device=DEV)
            lse = torch.empty((2, n), device=DEV)
            b = dqt.kv_batch(dev32(table), dev32([250]), n, 2, dev32([0, n]))
            dqt.dqt_kv_attn(h, b, Q.to(DEV), O, lse, dqt.workspace(dqt.dqt_kv_attn_workspace(h, b)))
            torch.cuda.synchronize()
            K, V, there = c.values(table[0], 250, 4)
            r = R.attention(Q, K, V, there, 0.125, True)
            assert ((O.double().cpu() - r["O"]).abs() <= r["t_O"]).all()
            assert ((lse.double().cpu() - r["lse"]).abs() <= r["t_lse"]).all()


def test_attention_nan_stays_in_its_sequence(lib):
    log("cache attention: NaN codes")
    gen = torch.Generator().manual_seed(6)
    c = random_cache(gen, 4, 2, 64, "e4m3")
    c.K[1, 0, 3, 3] = c.V[1, 0, 5, 7] = 0x7F
    h = device_cache(c)
    for n in (1, 60):
        Q = torch.randn((2 * n, 4, 64), generator=gen).to(torch.bfloat16).to(DEV)
        O = torch.empty_like(Q)
        b = dqt.kv_batch(dev32([[0, 1], [2, 3]]), dev32([100, 128]), 2 * n, 4, dev32([0, n, 2 * n]))
        dqt.dqt_kv_attn(h, b, Q, O, None, dqt.workspace(dqt.dqt_kv_attn_workspace(h, b)))
        torch.cuda.synchronize()
        assert torch.isnan(O[:n, :2]).any() and torch.isfinite(O[n:].float()).all() and torch.isfinite(O[:, 2:].float()).all()


def test_attention_one_row_of_nan_queries(lib):
    """A query of NaN gives NaN for itself alone."""
    log("cache attention: a NaN query")
    gen = torch.Generator().manual_seed(8)
    c = random_cache(gen, 8, 1, 64, "int8")
    h = device_cache(c)
    for n in (4, 70):
        Q = torch.randn((n, 2, 64), generator=gen).to(torch.bfloat16)
        Q[2, 1, 9] = float("nan")
        O = torch.empty((n, 2, 64), dtype=torch.bfloat16, device=DEV)
        b = dqt.kv_batch(dev32([list(range(8))]), dev32([500]), n, 2, dev32([0, n]))
        dqt.dqt_kv_attn(h, b, Q.to(DEV), O, None, dqt.workspace(dqt.dqt_kv_attn_workspace(h, b)))
        torch.cuda.synchronize()
        bad = torch.isnan(O.float()).any(-1).cpu()
        want = torch.zeros_like(bad)
        want[2, 1] = True
        assert torch.equal(bad, want)


def test_attention_far_pages(lib):
    """Pages whose bytes lie past 2^31 and 2^32."""
    log("cache attention and append: pages past 2^32 bytes")
    kvh, d = 16, 128
    pages = (1 << 32) // (kvh * R.PAGE * d) + 40
    gen = torch.Generator().manual_seed(7)
    small = random_cache(gen, 3, kvh, d, "int8")
    K = torch.zeros((pages, kvh, R.PAGE, d), dtype=torch.int8, device=DEV)
    V = torch.zeros((pages, kvh, d, R.PAGE), dtype=torch.int8, device=DEV)
    scales = torch.ones((pages, kvh, 2), device=DEV)
    far = [pages - 1, pages // 2 + 3, pages - 17]
    for i, p in enumerate(far):
        K[p], V[p], scales[p] = small.K[i].view(torch.int8).to(DEV), small.V[i].view(torch.int8).to(DEV), small.scales[i].to(DEV)
    h = dqt.KvCache(K, V, scales)
    kn, vn = (torch.randn((1, kvh, d), generator=gen).to(torch.bfloat16) for _ in range(2))
    b = dqt.kv_batch(dev32([far]), dev32([150]), 1, kvh)
    dqt.dqt_kv_append(h, b, kn.to(DEV), vn.to(DEV))
    small.write([0, 1, 2], 149, kn.float(), vn.float())
    Q = torch.randn((1, kvh, d), generator=gen).to(torch.bfloat16)
    O = torch.empty((1, kvh, d), dtype=torch.bfloat16, device=DEV)
    dqt.dqt_kv_attn(h, b, Q.to(DEV), O, None, dqt.workspace(dqt.dqt_kv_attn_workspace(h, b)))
    dqt.dqt_kv_copy([h], [far[2]], [1])
    torch.cuda.synchronize()
    k, v, there = small.values([0, 1, 2], 150, 3)
    r = R.attention(Q, k, v, there, d ** -0.5, True)
    assert ((O.double().cpu() - r["O"]).abs() <= r["t_O"]).all()
    for p in (far[2], 1):
        assert torch.equal(K[p].cpu(), small.K[2].view(torch.int8)) and torch.equal(V[p].cpu(), small.V[2].view(torch.int8))
        assert torch.equal(scales[p].cpu(), small.scales[2])


# ------------------------------------------------------------------ pages

@pytest.mark.parametrize("fmt,d,kvh,layers,pages,n", [("e4m3", 64, 1, 1, 2, 1), ("int8", 128, 3, 5, 40, 20),
                                                      ("int8", 64, 2, 2, 1200, 600), ("e4m3", 64, 1, 40, 9, 4),
                                                      ("e4m3", 64, 1, 1, 70000, 300)])
def test_copy(lib, fmt, d, kvh, layers, pages, n):
    log(f"copy {fmt} d={d} kv_heads={kvh} layers={layers} pages={pages} n={n}")
    rng, gen = np.random.default_rng(n), torch.Generator().manual_seed(n)
    caches, want = [], []
    for _ in range(layers):
        k = torch.randint(0, 256, (pages, kvh, R.PAGE, d), generator=gen, dtype=torch.uint8).to(DEV)
        v = torch.randint(0, 256, (pages, kvh, d, R.PAGE), generator=gen, dtype=torch.uint8).to(DEV)
        s = torch.rand((pages, kvh, 2), generator=gen).to(DEV)
        want.append([x.clone() for x in (k, v, s)])
        caches.append(dqt.KvCache(k.view(R.DTYPE[fmt]), v.view(R.DTYPE[fmt]), s))
    order = rng.permutation(pages)
    src, dst = order[:n].copy(), order[n:2 * n]
    src[-1] = src[0]                                  # (a page may be copied twice)
    dqt.dqt_kv_copy(caches, src, dst)
    torch.cuda.synchronize()
    a, b = (torch.as_tensor(x).to(DEV) for x in (src, dst))
    for c, w in zip(caches, want):
        for x, y in zip((c.K.view(torch.uint8), c.V.view(torch.uint8), c.scales), w):
            y[b] = y[a]
            assert torch.equal(x, y)


# ------------------------------------------------------------------ together

@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
def test_decoding(lib, fmt):
    """Prompts, single tokens, a fork whose branches go apart, drafts that are dropped, a
    sequence that ends, a compaction: at every step the attention is that of the cache's
    contents in 64 bits, and near that of the keys and values that were given."""
    log(f"decoding {fmt}")
    heads, kvh, d, rot = 6, 2, 64, 64
    gen = torch.Generator().manual_seed(11)
    pool = dqt.KvPool(24, 4, 6)
    h = dqt.kv_cache(24, kvh, d, FMT[fmt])
    rope = dqt.rope(d, rot)
    f = dqt.dqt_rope_freqs(rot)
    full = [[torch.zeros((0, kvh, d)), torch.zeros((0, kvh, d))] for _ in range(4)]    # what each sequence was given

    def copies(pairs):
        dqt.dqt_kv_copy([h], *pairs)

    def step(lq):
        """New tokens for the sequences of lq, in one append and one attention."""
        seqs = sorted(lq)
        for s in seqs:
            copies(pool.extend(s, int(pool.len[s]) + lq[s]))
        n = [lq[s] for s in seqs]
        Q, K, V = (torch.randn((sum(n), x, d), generator=gen).to(torch.bfloat16) for x in (heads, kvh, kvh))
        b = dqt.kv_batch(dev32(pool.table[seqs]), dev32(pool.len[seqs]), sum(n), heads,
                         None if set(n) == {1} else dev32(starts(n)))
        Qr = torch.empty((sum(n), heads, d), dtype=torch.bfloat16, device=DEV)
        O, lse = torch.empty_like(Qr), torch.empty((heads, sum(n)), device=DEV)
        dqt.dqt_kv_append(h, b, K.to(DEV), V.to(DEV), rope, Q.to(DEV), Qr)
        dqt.dqt_kv_attn(h, b, Qr, O, lse, dqt.workspace(dqt.dqt_kv_attn_workspace(h, b)))
        torch.cuda.synchronize()
        c = R.Cache(24, kvh, d, fmt, 0)
        c.K, c.V, c.scales = h.K.view(torch.uint8).cpu(), h.V.view(torch.uint8).cpu(), h.scales.cpu()
        at = 0
        for s, m in zip(seqs, n):
            rows, at = slice(at, at + m), at + m
            pos = np.arange(pool.len[s] - m, pool.len[s])
            full[s] = [torch.cat((x, y)) for x, y in zip(full[s], (R.rotate(K[rows], pos, f, rot, False)[0], V[rows].double()))]
            k, v, there = c.values(pool.table[s], int(pool.len[s]), 24)
            q = Qr[rows].double().cpu()
            r = R.attention(q, k, v, there, d ** -0.5, True)
            assert ((O[rows].double().cpu() - r["O"]).abs() <= r["t_O"]).all(), (s, m)
            assert ((lse[:, rows].double().cpu() - r["lse"]).abs() <= r["t_lse"]).all()
            # with s the page's scale now: an e4m3 value is off by 2^-4 of itself, below 2^-6 s by half a step of
            # 2^-9 s, again (on half the step each time before) where s grew: 2^-9 s in all; an int8 value by
            # s / 2 + s / 4 + ... < s.  The rotation's fp32 roundings add 4 F32 (|a| + |b|), below 2^-19 here.
            page = torch.as_tensor(pool.table[s][np.arange(pool.len[s]) // R.PAGE].astype(np.int64))
            for j, (x, y) in enumerate(((full[s][0], k), (full[s][1], v))):
                sc = c.scales[page, :, j].double()[..., None]
                err = 2.0 ** -4 * x.abs() + 2.0 ** -9 * sc if fmt == "e4m3" else sc
                assert ((x - y).abs() <= err + 2.0 ** -19).all(), (s, float((x - y).abs().max()))

    step({0: 100, 1: 3, 2: 64})
    for _ in range(4):
        step({0: 1, 1: 1, 2: 1})
    pool.fork(0, 3)
    full[3] = list(full[0])
    for _ in range(3):
        step({0: 1, 1: 1, 2: 1, 3: 1})
    step({0: 5, 3: 2, 1: 1})                          # drafts of sequence 0, of which two are kept
    pool.trim(0, int(pool.len[0]) - 3)
    full[0] = [x[:-3] for x in full[0]]
    step({0: 1, 1: 62, 3: 30})
    pool.trim(2)
    full[2] = [x[:0] for x in full[2]]
    copies(pool.compact())
    assert pool.table.max() < 24 - pool.n_free
    for _ in range(3):
        step({0: 1, 1: 1, 3: 1})
    step({2: 70, 0: 1})


@pytest.mark.parametrize("width,split", [(20, False), (150, True)])
def test_decoding_captured(lib, width, split):
    """Append and attention captured once, replayed while the lengths move on the device;
    eager calls of the same kind between the replays."""
    log(f"decoding captured {width}")
    heads, kvh, d, n = 4, 2, 64, 3
    gen = torch.Generator().manual_seed(12)
    table = dev32(np.random.default_rng(1).permutation(n * width).reshape(n, width))
    kv_len = dev32([60, 1, 64 * width - 82])
    caches = [dqt.kv_cache(n * width, kvh, d, dqt.DQT_I8) for _ in range(2)]
    for x in ("K", "V", "scales"):
        getattr(caches[0], x).copy_((torch.rand(getattr(caches[0], x).shape, generator=gen) * 40).to(getattr(caches[0], x).dtype))
        if x == "scales":
            caches[0].scales.fill_(2.0 ** -5)
        getattr(caches[1], x).copy_(getattr(caches[0], x))
    rope = dqt.rope(d)
    Q, K, V = (torch.randn((n, x, d), generator=gen).to(torch.bfloat16).to(DEV) for x in (heads, kvh, kvh))
    out = [[torch.empty_like(Q), torch.empty_like(Q), torch.empty((heads, n), device=DEV)] for _ in range(2)]
    b = dqt.kv_batch(table, kv_len, n, heads)
    ws = [dqt.workspace(dqt.dqt_kv_attn_workspace(caches[0], b)) for _ in range(2)]
    assert (ws[0] is not None) == split               # (the keys are split over blocks)

    def run(i):
        dqt.dqt_kv_append(caches[i], b, K, V, rope, Q, out[i][0])
        dqt.dqt_kv_attn(caches[i], b, out[i][0], out[i][1], out[i][2], ws[i])

    s, g = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(g, stream=s):
        run(0)
    torch.cuda.current_stream().wait_stream(s)
    for k in range(6):
        K.copy_(torch.randn(K.shape, generator=gen) * (k + 1))
        V.copy_(torch.randn(V.shape, generator=gen))
        g.replay()
        run(1)
        torch.cuda.synchronize()
        for x, y in zip(out[0] + [caches[0].K, caches[0].V, caches[0].scales], out[1] + [caches[1].K, caches[1].V, caches[1].scales]):
            assert torch.equal(x, y), k
        kv_len.add_(1 if k != 2 else -2)


def test_bit_reproducible_and_streams(lib):
    """Two streams with workspaces of their own give the bits of one call."""
    log("cache attention: streams")
    gen = torch.Generator().manual_seed(13)
    c = random_cache(gen, 200, 4, 128, "e4m3")
    h = device_cache(c)
    table, lens = dev32(np.arange(200).reshape(2, 100)), dev32([6400, 3333])
    Q = torch.randn((2, 16, 128), generator=gen).to(torch.bfloat16).to(DEV)
    b = dqt.kv_batch(table, lens, 2, 16)
    O = [torch.empty_like(Q) for _ in range(3)]
    ws = [dqt.workspace(dqt.dqt_kv_attn_workspace(h, b)) for _ in range(3)]
    ss = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    for _ in range(3):
        for i, s in enumerate(ss):
            dqt.dqt_kv_attn(h, b, Q, O[i], None, ws[i], stream=s)
    dqt.dqt_kv_attn(h, b, Q, O[2], None, ws[2])
    torch.cuda.synchronize()
    assert torch.equal(O[0], O[2]) and torch.equal(O[1], O[2])
