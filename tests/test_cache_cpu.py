"""Rotary positions, the 8-bit cache and its pages without a GPU: argument checks
(every refusal comes before anything is launched), the frequencies, and who holds
which page."""
import ctypes
import math
from fractions import Fraction

import numpy as np
import pytest
import torch

from paper_2412_04787_amd import dqt

FAKE, ODD = 1 << 20, (1 << 20) + 4
S, N, A, D, R, W = (dqt.DQT_ERR_SHAPE, dqt.DQT_ERR_NULL, dqt.DQT_ERR_ALIGN, dqt.DQT_ERR_DTYPE, dqt.DQT_ERR_RANGE,
                    dqt.DQT_ERR_WORKSPACE)
INF, NAN = float("inf"), float("nan")


def make(kind, base, kw):
    d = dict(base, **kw)
    return kind(*[d[n] for n, _ in kind._fields_])


def cache(**kw):
    return make(dqt.DqtKvCache, dict(K=FAKE, V=FAKE, scales=FAKE, pages=100, kv_heads=2, d=64, fmt=dqt.DQT_FP8E4M3, reserved=0), kw)


def batch(**kw):
    return make(dqt.DqtKvBatch, dict(table=FAKE, kv_len=FAKE, q_start=FAKE, q_tokens=8, max_len=640, n_seq=4, table_stride=10,
                                     heads=8, causal=1, scale=0.125, reserved=0), kw)


def rows(p=FAKE, token=1024, head=128):
    return dqt.DqtRows(p, token, head)


def rope(**kw):
    return make(dqt.DqtRope, dict(freq=FAKE, d=64, rot=64, pairs=0, reserved=0, amp=1.0), kw)


def by(x):
    return None if x is None else ctypes.byref(x)


def append(c=None, b=None, k=rows(), v=rows(), r=None, q=None, qr=None):
    return dqt.load().dqt_kv_append(by(c or cache()), by(b or batch()), by(k), by(v), by(r), by(q), by(qr), None)


def attn(c=None, b=None, q=rows(), o=rows(), lse=FAKE, ws=FAKE, nbytes=1 << 40):
    return dqt.load().dqt_kv_attn(by(c or cache()), by(b or batch()), by(q), by(o), lse, ws, nbytes, None)


def test_struct_layouts():
    assert ctypes.sizeof(dqt.DqtRope) == 32 and dqt.DqtRope.amp.offset == 24
    assert ctypes.sizeof(dqt.DqtRopeIO) == 56 and dqt.DqtRopeIO.heads.offset == 48
    assert ctypes.sizeof(dqt.DqtKvCache) == 48 and dqt.DqtKvCache.pages.offset == 24
    assert ctypes.sizeof(dqt.DqtKvBatch) == 64 and dqt.DqtKvBatch.scale.offset == 56
    assert ctypes.sizeof(dqt.DqtKvPool) == 24


@pytest.mark.parametrize("kw,status", [
    (dict(pages=-1), S), (dict(pages=1 << 31), S), (dict(kv_heads=0), S), (dict(kv_heads=1025), S), (dict(d=96), S),
    (dict(d=256), S), (dict(fmt=dqt.DQT_BF16), D), (dict(fmt=dqt.DQT_INT4), D), (dict(reserved=1), R), (dict(K=None), N),
    (dict(V=None), N), (dict(scales=None), N), (dict(K=FAKE + 8), A), (dict(V=ODD), A), (dict(scales=ODD), A),
])
def test_cache_descriptor(kw, status):
    c = cache(**kw)
    assert append(c) == status and attn(c) == status
    assert dqt.load().dqt_kv_attn_workspace(by(c), by(batch())) == 0
    one = np.array([1], np.int32)
    assert dqt.load().dqt_kv_copy(1, by(c), 1, one.ctypes.data, np.array([2], np.int32).ctypes.data, None) == status


@pytest.mark.parametrize("kw,status", [
    (dict(table=None), N), (dict(kv_len=None), N), (dict(q_start=None), S), (dict(q_tokens=-1), S), (dict(q_tokens=1 << 31), S),
    (dict(q_tokens=1 << 28), S), (dict(max_len=-1), S), (dict(max_len=641), S), (dict(n_seq=-1), S), (dict(n_seq=0), S),
    (dict(table_stride=-1), S), (dict(heads=0), S), (dict(heads=3), S), (dict(heads=1026), S), (dict(causal=2), R),
    (dict(scale=0.0), R), (dict(scale=NAN), R), (dict(scale=INF), R), (dict(reserved=3), R), (dict(table=FAKE + 2), A),
    (dict(kv_len=FAKE + 1), A), (dict(q_start=FAKE + 2), A), (dict(n_seq=1 << 23), S),
    (dict(max_len=1 << 31, table_stride=1 << 26), S),
])
def test_batch_descriptor(kw, status):
    b = batch(**kw)
    assert append(b=b) == status and attn(b=b) == status
    assert dqt.load().dqt_kv_attn_workspace(by(cache()), by(b)) == 0


def test_append_and_attention_arguments():
    lib = dqt.load()
    assert lib.dqt_kv_append(None, by(batch()), by(rows()), by(rows()), None, None, None, None) == N
    assert lib.dqt_kv_attn(by(cache()), None, by(rows()), by(rows()), None, FAKE, 1 << 40, None) == N
    bad_in = [(None, N), (rows(p=None), N), (rows(p=ODD), A), (rows(token=1028), A), (rows(head=4), A), (rows(token=-8), S),
              (rows(token=(1 << 23) + 8), S), (rows(head=(1 << 40) + 8), S)]
    bad_out = bad_in[1:] + [(rows(token=0), S), (rows(head=0), S), (rows(token=512), S), (rows(token=64, head=64), S)]
    other = rows(p=1 << 21)
    for x, st in bad_in:
        assert append(k=x) == st and append(v=x) == st and attn(q=x) == st
        if x is not None:
            assert append(r=rope(), q=x, qr=other) == st
    for x, st in bad_out:
        assert attn(o=x) == st and append(r=rope(), q=other, qr=x) == st
    assert append(q=rows(), qr=other) == N                     # rotated queries without a rotation
    assert append(r=rope(), q=rows()) == N and append(r=rope(), qr=rows()) == N
    assert append(r=rope(), q=rows(), qr=rows(token=2048)) == S          # in place, other strides
    assert append(r=rope(d=128)) == S
    assert attn(lse=FAKE + 2) == A and attn(ws=ODD) == A
    long = batch(max_len=64 * 10000, table_stride=10000)
    need = lib.dqt_kv_attn_workspace(by(cache()), by(long))
    assert need > 0 and attn(b=long, ws=None) == W and attn(b=long, nbytes=need - 1) == W
    assert lib.dqt_kv_attn_workspace(by(cache()), by(batch())) >= 0
    # nothing to do: no launch
    none = batch(q_tokens=0, n_seq=0, q_start=None, table=None, kv_len=None, max_len=0, table_stride=0)
    assert append(b=none, k=rows(p=None), v=rows(p=None)) == 0 and attn(b=none, q=rows(p=None), o=rows(p=None), ws=None, nbytes=0) == 0


@pytest.mark.parametrize("kw,status", [
    (dict(freq=None), N), (dict(freq=ODD), A), (dict(d=8, rot=8), S), (dict(d=72), S), (dict(d=1040), S), (dict(rot=0), S),
    (dict(rot=24), S), (dict(rot=80), S), (dict(rot=-16), S), (dict(pairs=2), R), (dict(reserved=1), R), (dict(amp=NAN), R),
    (dict(amp=INF), R),
])
def test_rope_descriptor(kw, status):
    r = rope(**kw)
    io = dqt.DqtRopeIO(rows(), rows(), 4, 0)
    for fn in (dqt.load().dqt_rope_fwd, dqt.load().dqt_rope_bwd):
        assert fn(by(r), 1, by(io), dqt.DQT_BF16, 8, None, None) == status
    if "d" not in kw:                    # (the cache's heads are 64 wide)
        assert append(r=r) == status


def test_rope_arguments():
    io = lambda x=rows(), y=rows(p=1 << 21), heads=4, reserved=0: dqt.DqtRopeIO(x, y, heads, reserved)
    for fn in (dqt.load().dqt_rope_fwd, dqt.load().dqt_rope_bwd):
        call = lambda x, n=1, t=dqt.DQT_F32, tokens=8, pos=None, r=rope(): fn(by(r), n, by(x), t, tokens, pos, None)
        assert call(io(), r=None) == N and call(None) == N
        assert call(io(), n=0) == S and call(io(), n=5) == S
        assert call(io(), t=dqt.DQT_I8) == D
        assert call(io(), tokens=-1) == S and call(io(), tokens=1 << 31) == S and call(io(), tokens=1 << 30) == S
        assert call(io(), pos=FAKE + 2) == A
        assert call(io(heads=0)) == S and call(io(heads=1025)) == S and call(io(reserved=1)) == R
        assert call(io(x=rows(p=None))) == N and call(io(y=rows(p=None))) == N
        assert call(io(x=rows(p=ODD))) == A and call(io(y=rows(head=4))) == A
        assert call(io(y=rows(token=0))) == S and call(io(y=rows(p=1 << 21, token=128))) == S
        assert call(io(y=rows(token=2048))) == S                # in place, other strides
        assert call(io(), tokens=0) == 0


def test_rope_freqs_values():
    """round(2^64 base^(-2 i / rot) / 2 pi) by exact fractions; blended for stretched contexts."""
    pi = Fraction(3141592653589793238462643383279502884197169399375105820974944592307816, 10 ** 69)
    for rot, base in ((16, 16.0), (128, 10000.0), (64, 500000.0)):
        f = dqt.dqt_rope_freqs(rot, base)
        assert f.dtype == np.uint64 and f.shape == (rot // 2,)
        for i in range(rot // 2):
            # base^(-2 i / rot) to 2^-100, by the integer root of a scaled power
            n, k = rot // 2, 400
            g = math.gcd(i, n) or n
            num, den = i // g, n // g
            x = (1 << (k * den)) // int(base) ** num
            lo, hi = 0, 1 << (k + 1)
            while hi - lo > 1:
                mid = (lo + hi) // 2
                lo, hi = (mid, hi) if mid ** den <= x else (lo, mid)
            want = Fraction(lo, 1 << k) / (2 * pi) * (1 << 64)
            # (long double: 64 bits, a power, a quotient)
            assert abs(int(f[i]) - want) <= 1 + want / (1 << 60), (rot, i)
    plain = dqt.dqt_rope_freqs(64, 10000.0).astype(np.float64)
    turns = 4096 * plain / 2.0 ** 64
    for factor, slow, fast in ((8.0, 1.0, 4.0), (4.0, 1.0, 32.0), (2.0, 0.0, 0.0), (3.0, 5.0, 5.0)):
        f = dqt.dqt_rope_freqs(64, 10000.0, factor, 4096.0, slow, fast).astype(np.float64)
        k = np.clip((turns - slow) / (fast - slow), 0, 1) if fast > slow else 0.0
        # (f and plain are each rounded to a whole number: 1/2 + 1/2; doubles add some 2^-50 of the value)
        np.testing.assert_allclose(f, plain * (k + (1 - k) / factor), rtol=1e-14, atol=1.0)
    for bad in (dict(base=1.0), dict(base=NAN), dict(base=INF), dict(factor=0.5), dict(factor=INF), dict(context=-1.0),
                dict(slow=-1.0), dict(slow=3.0, fast=2.0), dict(fast=INF), dict(slow=NAN)):
        with pytest.raises(dqt.DqtError) as e:
            dqt.dqt_rope_freqs(64, **bad)
        assert e.value.status == R
    for rot in (0, 8, 20, 1040, -16):
        with pytest.raises(dqt.DqtError) as e:
            dqt.dqt_rope_freqs(rot)
        assert e.value.status == S


def test_copy_refusals():
    lib = dqt.load()
    arr = (dqt.DqtKvCache * 2)(cache(), cache())
    i32 = lambda *x: np.array(x, np.int32)

    def call(src, dst, n=None, caches=arr, m=2):
        return lib.dqt_kv_copy(m, caches, len(src) if n is None else n, src.ctypes.data, dst.ctypes.data, None)

    assert call(i32(0), i32(100)) == R and call(i32(-1), i32(1)) == R and call(i32(100), i32(1)) == R and call(i32(0), i32(-1)) == R
    assert call(i32(0, 1), i32(5, 5)) == R                       # twice the same destination
    assert call(i32(0, 1), i32(1, 2)) == R and call(i32(3), i32(3)) == R          # read and written
    assert call(i32(0), i32(1), n=-1) == S and call(i32(0), i32(1), m=-1) == S
    assert lib.dqt_kv_copy(2, arr, 1, None, i32(1).ctypes.data, None) == N
    assert lib.dqt_kv_copy(1, None, 1, i32(0).ctypes.data, i32(1).ctypes.data, None) == N
    for kw in (dict(pages=99), dict(kv_heads=1), dict(d=128), dict(fmt=dqt.DQT_I8)):
        assert call(i32(0), i32(1), caches=(dqt.DqtKvCache * 2)(cache(), cache(**kw))) == S
    many = (dqt.DqtKvCache * 1)(cache(pages=1 << 20))
    assert call(i32(0, 70000), i32(99999, 99999), caches=many, m=1) == R
    assert call(i32(0, 99999), i32(99999, 7), caches=many, m=1) == R
    assert call(i32(), i32()) == 0 and call(i32(0), i32(1), m=0) == 0


# ------------------------------------------------------------------ the binding

def test_binding_refuses_host_tensors_and_wrong_shapes():
    K, V = torch.zeros((2, 1, 64, 64), dtype=torch.int8), torch.zeros((2, 1, 64, 64), dtype=torch.int8)
    sc = torch.zeros((2, 1, 2))
    with pytest.raises(ValueError, match="host memory"):
        dqt.KvCache(K, V, sc)
    for bad in ((K[:, :, :32], V, sc), (K.float(), V, sc), (K, V[:1], sc), (K, V.view(torch.uint8), sc), (K, V, sc[..., :1]),
                (K, V, sc.double()), (K.transpose(2, 3), V, sc), (K[0], V, sc)):
        with pytest.raises(ValueError):
            dqt.KvCache(*bad)
    with pytest.raises(ValueError, match="host memory"):
        dqt.Rope(torch.zeros(32, dtype=torch.int64), 64)
    with pytest.raises(ValueError, match="host memory"):
        dqt.kv_batch(torch.zeros((2, 3), dtype=torch.int32), torch.zeros(2, dtype=torch.int32), 2, 4)


def test_binding_refuses_what_is_no_page():
    for bad in ([1 << 32], [-(1 << 40)], [1.0], np.array([1 << 35])):
        with pytest.raises(ValueError):
            dqt.dqt_kv_copy([], bad, [1])
    with pytest.raises(ValueError):
        dqt.dqt_kv_copy([], [1, 2], [3])


# ------------------------------------------------------------------ pages

def consistent(p, tables):
    """Free pages and holders agree with the tables."""
    count = np.zeros_like(p.refs)
    for x in tables.ravel():
        if x >= 0:
            count[x] += 1
    assert np.array_equal(count, p.refs)
    free = p.free_pages[:p.n_free]
    assert len(set(free.tolist())) == p.n_free and (p.refs[free] == 0).all() and p.n_free == (p.refs == 0).sum()


def test_pool_against_a_model():
    """Random extends, forks, trims and compactions against tokens kept in a plain
    array: every sequence finds its own tokens in its pages, no one else's."""
    rng = np.random.default_rng(5)
    for trial in range(6):
        pages, n, width = 40, 6, 9
        p = dqt.KvPool(pages, n, width)
        mem = np.full((pages, 64), -1, np.int64)
        text, fresh = [[] for _ in range(n)], 0

        def copy(pairs):
            src, dst = (np.asarray(x, np.int64) for x in pairs)
            assert not set(src) & set(dst) and len(set(dst)) == len(dst)
            mem[dst] = mem[src]

        for step in range(300):
            s, op = int(rng.integers(n)), rng.random()
            have = len(text[s])
            if op < 0.6:
                new = min(have + int(rng.integers(0, 90)), 64 * width)
                before = (p.table.copy(), p.refs.copy(), p.n_free)
                try:
                    copy(p.extend(s, new))
                except dqt.DqtError as e:
                    assert e.status == W and p.len[s] == have
                    assert np.array_equal(before[0], p.table) and np.array_equal(before[1], p.refs) and before[2] == p.n_free
                    continue
                for t in range(have, new):
                    mem[p.table[s, t // 64], t % 64] = fresh
                    text[s].append(fresh)
                    fresh += 1
            elif op < 0.75:
                to = int(rng.integers(n))
                if to != s and not text[to]:
                    p.fork(s, to)
                    text[to] = list(text[s])
            elif op < 0.95:
                new = 0 if rng.random() < 0.5 else int(rng.integers(0, have + 1))
                p.trim(s, new)
                text[s] = text[s][:new]
            else:
                copy(p.compact())
                assert (p.table < pages - p.n_free).all()
            consistent(p, p.table)
            for i in range(n):
                assert p.len[i] == len(text[i])
                assert [mem[p.table[i, t // 64], t % 64] for t in range(len(text[i]))] == text[i]
                assert (p.table[i, -(-len(text[i]) // 64):] == -1).all()


def test_pool_refusals():
    p = dqt.KvPool(4, 2, 3)
    lib, ref = dqt.load(), ctypes.byref(p.desc)
    row, x = p.table[0].ctypes.data, ctypes.byref(ctypes.c_int32())
    p.extend(0, 100)

    def status(f, *a):
        with pytest.raises(dqt.DqtError) as e:
            f(*a)
        return e.value.status

    assert status(p.extend, 0, 99) == S and status(p.extend, 0, 193) == S and status(p.trim, 0, 101) == S
    p.fork(0, 1)
    p.extend(0, 180)                      # a copy of the shared page, and one more
    assert p.n_free == 0 and status(p.extend, 1, 129) == W
    assert lib.dqt_kv_pool_extend(None, row, 3, 180, 181, x, x) == N
    assert lib.dqt_kv_pool_extend(ref, None, 3, 180, 181, x, x) == N
    assert lib.dqt_kv_pool_extend(ref, row, 3, 180, 181, None, x) == N
    assert lib.dqt_kv_pool_extend(ref, row, -1, 0, 0, x, x) == S and lib.dqt_kv_pool_extend(ref, row, 3, -1, 0, x, x) == S
    assert lib.dqt_kv_pool_fork(ref, row, 3, 180, row) == R and lib.dqt_kv_pool_fork(ref, row, 3, 180, None) == N
    assert lib.dqt_kv_pool_trim(ref, row, 3, 193, 0) == S
    bad = np.array([0, 0, 7], np.int32)
    assert lib.dqt_kv_pool_trim(ref, bad.ctypes.data, 3, 190, 0) == R               # page 7 of 4
    keep = p.refs.copy()
    bad[2] = p.table[1, 1]                # held once, listed with page 0 three times (held twice)
    bad[:2] = 0
    p.table[1] = -1
    assert p.refs[0] == 2
    assert lib.dqt_kv_pool_trim(ref, np.array([0, 0, 0], np.int32).ctypes.data, 3, 190, 0) == R
    assert np.array_equal(keep, p.refs)
    assert status(p.compact) == R         # a sequence's row is missing
    empty = dqt.KvPool(0, 1, 1)
    assert status(empty.extend, 0, 1) == W and empty.compact()[0].size == 0
    assert lib.dqt_kv_pool_init(None, 1, None, None) == N and lib.dqt_kv_pool_init(ref, -1, None, None) == S
    assert lib.dqt_kv_pool_init(ref, 1, None, None) == N
    with pytest.raises(ValueError):
        p.extend(2, 1)
    with pytest.raises(ValueError):
        p.fork(1, 0)
