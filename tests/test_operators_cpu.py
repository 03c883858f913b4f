"""Argument checks of the attention, SwiGLU and log-probability calls, without a
GPU: every refusal comes before anything is launched."""
import ctypes

import pytest
import torch

from paper_2412_04787_amd import dqt

FAKE, ODD = 1 << 20, (1 << 20) + 4
S, N, A, D, R, W, U = (dqt.DQT_ERR_SHAPE, dqt.DQT_ERR_NULL, dqt.DQT_ERR_ALIGN, dqt.DQT_ERR_DTYPE, dqt.DQT_ERR_RANGE,
                       dqt.DQT_ERR_WORKSPACE, dqt.DQT_ERR_UNSUPPORTED)


def desc(**kw):
    d = dict(q_start=FAKE, k_start=FAKE, q_tokens=256, k_tokens=256, n_seq=2, heads=8, kv_heads=2, d=64, scale=0.125,
             causal=1, reserved=0)
    d.update(kw)
    return dqt.DqtAttn(*[d[n] for n, _ in dqt.DqtAttn._fields_])


def rows(p=FAKE, token=1024, head=128):
    return dqt.DqtRows(p, token, head)


def fwd(a, q=None, k=None, v=None, o=None, lse=FAKE, ws=FAKE, nbytes=1 << 40):
    r = [ctypes.byref(x if x is not None else rows()) for x in (q, k, v, o)]
    return dqt.load().dqt_attn_fwd(ctypes.byref(a), *r, lse, ws, nbytes, None)


def bwd(a, bad=None, at=0, lse=FAKE, ws=FAKE, nbytes=1 << 40):
    r = [ctypes.byref(bad if bad is not None and i == at else rows()) for i in range(8)]
    return dqt.load().dqt_attn_bwd(ctypes.byref(a), *r[:4], lse, *r[4:], ws, nbytes, None)


def test_struct_layouts():
    assert ctypes.sizeof(dqt.DqtAttn) == 64 and dqt.DqtAttn.scale.offset == 48 and dqt.DqtAttn.reserved.offset == 56
    assert ctypes.sizeof(dqt.DqtRows) == 24 and ctypes.sizeof(dqt.DqtCkptIO) == 32


@pytest.mark.parametrize("kw,status", [
    (dict(d=32), S), (dict(d=96), S), (dict(d=256), S), (dict(heads=0), S), (dict(kv_heads=0), S),
    (dict(kv_heads=3), S), (dict(heads=2048, kv_heads=2048), S), (dict(n_seq=0), S), (dict(q_tokens=-1), S),
    (dict(k_tokens=-1), S), (dict(k_tokens=1 << 31), S), (dict(q_tokens=1 << 29), S), (dict(n_seq=1 << 23), S),
    (dict(q_start=None), N), (dict(k_start=None), N), (dict(q_start=FAKE + 2), A),
    (dict(scale=0.0), R), (dict(scale=-1.0), R), (dict(scale=float("nan")), R), (dict(scale=float("inf")), R),
    (dict(causal=2), R), (dict(reserved=1), R),
])
def test_attention_descriptor(kw, status):
    a = desc(**kw)
    assert fwd(a) == status and bwd(a) == status
    assert dqt.dqt_attn_fwd_workspace(a) == 0 and dqt.dqt_attn_bwd_workspace(a) == 0


def test_attention_arguments():
    lib = dqt.load()
    a = desc()
    assert lib.dqt_attn_fwd(None, *[ctypes.byref(rows())] * 4, FAKE, FAKE, 1 << 40, None) == N
    assert lib.dqt_attn_fwd(ctypes.byref(a), None, *[ctypes.byref(rows())] * 3, FAKE, FAKE, 1 << 40, None) == N
    bad_in = [(rows(p=None), N), (rows(p=ODD), A), (rows(token=1028), A), (rows(head=4), A), (rows(token=-8), S),
              (rows(token=(1 << 23) + 8), S), (rows(head=(1 << 40) + 8), S)]
    bad_out = bad_in + [(rows(token=0), S), (rows(head=0), S), (rows(token=512), S), (rows(token=64, head=64), S),
                        (rows(token=1024, head=32), S)]
    for x, st in bad_in:
        for n in "qkv":
            assert fwd(a, **{n: x}) == st
        for i in range(5):
            assert bwd(a, x, i) == st
    for x, st in bad_out:
        assert fwd(a, o=x) == st
        assert bwd(a, x, 5) == st
    # (dk, dv have 2 heads: a head stride of 128 and a token stride of 192 do not overlap)
    for i in (6, 7):
        assert bwd(a, rows(token=128), i) == S
        assert bwd(a, rows(token=184), i) == S
    assert fwd(a, lse=FAKE + 2) == A and bwd(a, lse=None) == N
    assert bwd(a, ws=None) == W and bwd(a, nbytes=dqt.dqt_attn_bwd_workspace(a) - 1) == W and bwd(a, ws=ODD) == A
    assert dqt.dqt_attn_bwd_workspace(a) >= 8 * 256 * 8


def test_attention_workspace_rule():
    """No workspace for a whole batch of prompts; a split of the keys for few
    rows over many keys, refused without its workspace."""
    assert dqt.dqt_attn_fwd_workspace(desc(q_tokens=16384, k_tokens=16384, n_seq=8, heads=16, kv_heads=16, d=128)) == 0
    assert dqt.dqt_attn_fwd_workspace(desc(q_tokens=37, k_tokens=37, n_seq=1, heads=4, kv_heads=4)) == 0
    a = desc(q_tokens=32, k_tokens=32 * 4096, n_seq=32, heads=32, kv_heads=8, d=128)
    need = dqt.dqt_attn_fwd_workspace(a)
    assert need > 0 and need % (32 * 32 * 129 * 4) == 0
    kw = dict(q=rows(token=4096), k=rows(token=1024), v=rows(token=1024), o=rows(token=4096))
    assert fwd(a, **kw, ws=None) == W and fwd(a, **kw, nbytes=need - 1) == W


def test_attention_nothing_to_do():
    """No query tokens: nothing is launched, whatever the other pointers are."""
    assert fwd(desc(q_tokens=0, k_tokens=0, n_seq=1, q_start=None, k_start=None), q=rows(p=None), k=rows(p=None),
               v=rows(p=None), o=rows(p=None), lse=None, ws=None, nbytes=0) == dqt.DQT_OK


def test_attention_tensors_checked_in_python():
    a = dqt.attn(4, 4, 2, 2, 64)
    t = torch.zeros((4, 2, 64), dtype=torch.bfloat16)
    for bad in (t.float(), t[:3], t[:, :1], torch.zeros((4, 64, 2), dtype=torch.bfloat16).transpose(1, 2)):
        with pytest.raises(ValueError):
            dqt.dqt_attn_fwd(a, t, t, bad, t)
    with pytest.raises(ValueError):
        dqt.attn(4, 4, 2, 2, 64, torch.zeros(2, dtype=torch.int64))
    with pytest.raises(ValueError):
        dqt.attn(4, 4, 2, 2, 64, torch.zeros(2, dtype=torch.int32), torch.zeros(3, dtype=torch.int32))


def ck(**kw):
    d = dict(Gq=FAKE, Uq=FAKE, gs=FAKE, us=FAKE)
    d.update(kw)
    return dqt.DqtCkptIO(d["Gq"], d["Uq"], d["gs"], d["us"])


def test_swiglu_arguments():
    lib = dqt.load()

    def f(G=FAKE, U=FAKE, t=dqt.DQT_BF16, M=4, K=64, act=dqt.DQT_I8, Xq=FAKE, xdq=FAKE, c=None):
        return lib.dqt_swiglu_act_quant(G, U, t, M, K, act, Xq, xdq, None if c is None else ctypes.byref(c), None)

    def b(dH=FAKE, t=dqt.DQT_BF16, G=FAKE, U=FAKE, c=None, M=4, K=64, dG=FAKE, dU=FAKE):
        return lib.dqt_swiglu_backward(dH, t, G, U, None if c is None else ctypes.byref(c), M, K, dG, dU, None)

    for kw, st in ((dict(M=-1), S), (dict(M=(1 << 28) + 1), S), (dict(K=0), S), (dict(K=24), S),
                   (dict(M=1 << 28, K=128), S)):
        assert f(**kw) == st and b(**kw) == st
    for kw, st in ((dict(t=dqt.DQT_I8), D), (dict(act=dqt.DQT_BF16), D), (dict(G=None), N), (dict(U=None), N),
                   (dict(Xq=None), N), (dict(xdq=None), N), (dict(G=ODD), A), (dict(U=ODD), A), (dict(Xq=ODD), A),
                   (dict(xdq=ODD), A), (dict(c=ck(Gq=None)), N), (dict(c=ck(us=None)), N), (dict(c=ck(Uq=ODD)), A),
                   (dict(c=ck(gs=ODD)), A)):
        assert f(**kw) == st, kw
    for kw, st in ((dict(t=dqt.DQT_I8), D), (dict(dH=None), N), (dict(dG=None), N), (dict(dU=None), N), (dict(G=None), N),
                   (dict(U=None), N), (dict(dH=ODD), A), (dict(dG=ODD), A), (dict(dU=ODD), A), (dict(G=ODD), A),
                   (dict(c=ck()), U), (dict(c=ck(gs=None), G=None, U=None), N)):
        assert b(**kw) == st, kw
    assert f(M=0, G=None, U=None, Xq=None, xdq=None) == dqt.DQT_OK
    assert b(M=0, dH=None, G=None, U=None, dG=None, dU=None) == dqt.DQT_OK


def test_logprob_arguments():
    lib = dqt.load()

    def f(X=FAKE, t=dqt.DQT_F32, M=4, V=100, st=100, tg=FAKE, lp=FAKE, lse=FAKE, en=FAKE, stat=FAKE, k=0, ids=None,
          tl=None, ws=None, nb=0):
        return lib.dqt_logprob_fwd(X, t, M, V, st, tg, lp, lse, en, stat, k, ids, tl, ws, nb, None)

    def b(X=FAKE, t=dqt.DQT_F32, M=4, V=100, st=100, tg=FAKE, stat=FAKE, en=FAKE, dl=FAKE, de=FAKE, dX=FAKE * 2, ds=100):
        return lib.dqt_logprob_bwd(X, t, M, V, st, tg, stat, en, dl, de, dX, ds, None)

    for kw, s in ((dict(M=-1), S), (dict(M=(1 << 23) + 1), S), (dict(V=0), S), (dict(V=(1 << 28) + 1, st=1 << 29, ), S),
                  (dict(st=99), S), (dict(t=dqt.DQT_I8), D), (dict(X=None), N), (dict(X=ODD), A), (dict(tg=ODD), A),
                  (dict(tg=None), N), (dict(stat=ODD), A), (dict(en=FAKE + 2), A)):
        assert f(**kw) == s and b(**kw) == s, kw
    for kw, s in ((dict(k=-1), S), (dict(k=33), S), (dict(k=3, V=2), S), (dict(k=3, ids=FAKE), N), (dict(k=3, tl=FAKE), N),
                  (dict(k=3, ids=ODD, tl=FAKE), A), (dict(lp=FAKE + 2), A), (dict(lse=FAKE + 2), A), (dict(ws=ODD), A)):
        assert f(**kw) == s, kw
    for kw, s in ((dict(stat=None), N), (dict(dX=None), N), (dict(en=None), N), (dict(dX=ODD), A), (dict(ds=99), S),
                  (dict(dl=FAKE + 2), A), (dict(de=FAKE + 2), A), (dict(X=FAKE, dX=FAKE, ds=104), S)):
        assert b(**kw) == s, kw
    # few rows of a large vocabulary are split and need a workspace
    need = dqt.dqt_logprob_workspace(2, 128000, 5)
    assert need > 0 and dqt.dqt_logprob_workspace(4096, 128000, 5) == 0 and dqt.dqt_logprob_workspace(2, 1000, 5) == 0
    big = dict(M=2, V=128000, st=128000, k=5, ids=FAKE, tl=FAKE)
    assert f(**big) == W and f(**big, ws=FAKE, nb=need - 1) == W
    assert f(M=0, X=None, tg=None, lp=None) == dqt.DQT_OK and b(M=0, X=None, stat=None, dX=None) == dqt.DQT_OK


def test_tensors_checked_in_python():
    x, y = torch.zeros((4, 64)), torch.zeros((4, 32))
    for args in ((x, y), (x, x.to(torch.bfloat16)), (x.t(), x.t())):
        with pytest.raises(ValueError):
            dqt.dqt_swiglu_act_quant(*args, dqt.DQT_I8, None, None)
    with pytest.raises(ValueError):
        dqt.dqt_logprob_fwd(x.t(), None, None)
    with pytest.raises(ValueError):
        dqt.dqt_logprob_bwd(x, None, None, None, y)


def test_tensors_of_another_device_are_refused(monkeypatch):
    class T:
        is_cuda = True

        def __init__(self, i):
            self.i = i

        def get_device(self):
            return self.i

    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 0, raising=False)
    dqt._here(T(0))
    with pytest.raises(ValueError):
        dqt._here(T(1))


class _Calls:
    """Stands for the library: counts the calls that reach it."""

    def __init__(self):
        self.n = 0

    def __getattr__(self, name):
        def call(*args):
            self.n += 1
            return dqt.DQT_OK
        return call


def _calls_of_each_operator():
    """(name, call, its tensors by name); the call takes the same tensors."""
    f32, bf16 = torch.float32, torch.bfloat16
    M, K, V, k = 3, 160, 50, 4
    f = lambda *s, dt=f32: torch.zeros(s, dtype=dt)
    i8 = torch.int8
    ck = lambda t: dqt.SwigluCkpt(t["Gq"], t["Uq"], t["gs"], t["us"])
    ckt = lambda: dict(Gq=f(M, K, dt=i8), Uq=f(M, K, dt=i8), gs=f(M, 2), us=f(M, 2))
    T, H, KV, D = 5, 4, 2, 64
    q, kv = lambda: f(T, H, D, dt=bf16), lambda: f(T, KV, D, dt=bf16)
    st = lambda: torch.tensor([0, T], dtype=torch.int32)
    desc = lambda t: dqt.attn(T, T, H, KV, D, t["q_start"], t["k_start"])
    return [
        ("swiglu", lambda t: dqt.dqt_swiglu_act_quant(t["G"], t["U"], dqt.DQT_I8, t["Xq"], t["xdq"], ck(t)),
         dict(G=f(M, K), U=f(M, K), Xq=f(M, K, dt=i8), xdq=f(M), **ckt())),
        ("swiglu backward", lambda t: dqt.dqt_swiglu_backward(t["dH"], t["G"], t["U"], t["dG"], t["dU"]),
         dict(dH=f(M, K), G=f(M, K), U=f(M, K), dG=f(M, K), dU=f(M, K))),
        ("swiglu backward ckpt", lambda t: dqt.dqt_swiglu_backward_ckpt(t["dH"], ck(t), t["dG"], t["dU"]),
         dict(dH=f(M, K), dG=f(M, K), dU=f(M, K), **ckt())),
        ("logprob", lambda t: dqt.dqt_logprob_fwd(t["X"], t["targets"], t["logp"], t["lse"], t["entropy"], t["stat"],
                                                  t["top_ids"], t["top_logp"], t["ws"]),
         dict(X=f(M, V), targets=f(M, dt=torch.int64), logp=f(M), lse=f(M), entropy=f(M), stat=f(M, 2),
              top_ids=f(M, k, dt=torch.int64), top_logp=f(M, k), ws=f(8))),
        ("logprob backward", lambda t: dqt.dqt_logprob_bwd(t["X"], t["targets"], t["stat"], t["dlogp"], t["dX"],
                                                           t["entropy"], t["dent"]),
         dict(X=f(M, V), targets=f(M, dt=torch.int64), stat=f(M, 2), dlogp=f(M), dX=f(M, V), entropy=f(M), dent=f(M))),
        ("attention", lambda t: dqt.dqt_attn_fwd(desc(t), t["Q"], t["K"], t["V"], t["O"], t["lse"], t["ws"]),
         dict(Q=q(), K=kv(), V=kv(), O=q(), lse=f(H, T), ws=f(8), q_start=st(), k_start=st())),
        ("attention backward", lambda t: dqt.dqt_attn_bwd(desc(t), t["Q"], t["K"], t["V"], t["O"], t["lse"], t["dO"],
                                                          t["dQ"], t["dK"], t["dV"], t["ws"]),
         dict(Q=q(), K=kv(), V=kv(), O=q(), lse=f(H, T), dO=q(), dQ=q(), dK=kv(), dV=kv(), ws=f(8), q_start=st(),
              k_start=st())),
    ]


OPERATORS = _calls_of_each_operator()


class _On:
    """A tensor of host memory that says it is on device i."""

    def __init__(self, t, i):
        self._t, self._i = t, i

    def get_device(self):
        return self._i

    is_cuda = True

    def __getattr__(self, name):
        return getattr(self._t, name)


@pytest.fixture
def calls(monkeypatch):
    c = _Calls()
    monkeypatch.setattr(dqt, "load", lambda: c)
    monkeypatch.setattr(dqt, "_stream", lambda stream=None: None)
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 0, raising=False)
    return c


@pytest.mark.parametrize("at", range(len(OPERATORS)), ids=[o[0] for o in OPERATORS])
def test_every_tensor_of_a_call_has_to_be_on_the_current_device(calls, at):
    name, call, tensors = OPERATORS[at]
    here = {n: _On(t, 0) for n, t in tensors.items()}
    call(here)
    assert calls.n == 1
    for n, t in tensors.items():
        for i in (-1, 1):                  # (-1: host memory)
            with pytest.raises(ValueError):
                call({**here, n: _On(t, i)})
    with pytest.raises(ValueError):
        call({n: _On(t, 1) for n, t in tensors.items()})
    with pytest.raises(ValueError):
        call(tensors)                      # all in host memory
    assert calls.n == 1


def _wrong(n, t):
    """Tensors that the call must not take for t: another type, one row fewer,
    one column fewer, not contiguous (where rows may have any stride: columns)."""
    other = {torch.float32: torch.float64, torch.int64: torch.int32, torch.int32: torch.int64, torch.int8: torch.int16,
             torch.bfloat16: torch.float16}[t.dtype]
    out = [] if n == "ws" else [t.to(other), t[:-1]]
    if t.dim() > 1:
        out.append(t[:, :-1])
        out.append(torch.zeros(t.shape[::-1], dtype=t.dtype).permute(*range(t.dim())[::-1]))
    else:
        out.append(torch.zeros((t.numel(), 2), dtype=t.dtype)[:, 0])
    return out


@pytest.mark.parametrize("at", range(len(OPERATORS)), ids=[o[0] for o in OPERATORS])
def test_every_tensor_of_a_call_has_its_type_size_and_strides(calls, at):
    name, call, tensors = OPERATORS[at]
    here = {n: _On(t, 0) for n, t in tensors.items()}
    for n, t in tensors.items():
        for i, bad in enumerate(_wrong(n, t)):
            if name.startswith("logprob") and n == "X" and i == 2 and "dX" not in tensors:
                continue                   # (fewer columns: another vocabulary)
            with pytest.raises((ValueError, KeyError)):
                call({**here, n: _On(bad, 0)})
                raise AssertionError((name, n, bad.dtype, tuple(bad.shape), bad.stride()))
    assert calls.n == 0


def test_larger_outputs_are_taken(calls):
    """Buffers of a larger batch serve a smaller one."""
    for name, call, tensors in OPERATORS:
        here = {n: _On(torch.zeros((t.shape[0] + 2, *t.shape[1:]), dtype=t.dtype), 0)
                if n in ("Xq", "xdq", "logp", "lse", "entropy", "stat", "top_ids", "top_logp", "ws") else _On(t, 0)
                for n, t in tensors.items()}
        call(here)
    assert calls.n == len(OPERATORS)


def test_targets_are_as_many_as_rows(calls):
    name, call, tensors = OPERATORS[3]
    with pytest.raises(ValueError):
        call({**{n: _On(t, 0) for n, t in tensors.items()}, "targets": _On(torch.zeros(4, dtype=torch.int64), 0)})
    assert calls.n == 0


def test_swiglu_gradients_are_two_buffers():
    """dG or dU may be dH's buffer, not both: one would overwrite the other."""
    lib, other, third = dqt.load(), FAKE * 2, FAKE * 3
    c = ck()
    for dG, dU in ((FAKE, FAKE), (other, other)):
        assert lib.dqt_swiglu_backward(FAKE, dqt.DQT_BF16, third, third, None, 4, 64, dG, dU, None) == S
        assert lib.dqt_swiglu_backward(FAKE, dqt.DQT_BF16, None, None, ctypes.byref(c), 4, 64, dG, dU, None) == S
    assert lib.dqt_swiglu_backward(FAKE, dqt.DQT_BF16, FAKE, FAKE, None, 0, 64, FAKE, FAKE, None) == dqt.DQT_OK


def test_alignment_of_vectors_of_one_value_a_row():
    """xdq 16 bytes as every other base, the rest its type's: a call with those
    is refused for its missing workspace, not for them."""
    lib = dqt.load()
    assert lib.dqt_act_quant(FAKE, dqt.DQT_BF16, 4, 64, dqt.DQT_I8, FAKE, ODD, None) == A
    assert lib.dqt_swiglu_act_quant(FAKE, FAKE, dqt.DQT_BF16, 4, 64, dqt.DQT_I8, FAKE, ODD, None, None) == A
    ids = FAKE + 8
    assert lib.dqt_logprob_fwd(FAKE, dqt.DQT_F32, 2, 128000, 128000, ids, ODD, ODD, ODD, ids, 5, ids, ODD, None, 0,
                               None) == W
    assert bwd(desc(), lse=ODD, ws=None) == W
