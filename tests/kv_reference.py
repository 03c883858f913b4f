"""Plain float64 implementations of rotary positions and of the 8-bit cache of keys
and values, written from their formulas, with bounds of what rounding may add.  A
rounding is off by at most half a step: 2^-8 of the value for bf16, 2^-11 for fp16,
2^-24 for fp32, 2^-4 for e4m3."""
import numpy as np
import torch

BF16, F16, F32 = 2.0 ** -8, 2.0 ** -11, 2.0 ** -24
PAGE = 64
TOP = {"e4m3": 448.0, "int8": 127.0}
DTYPE = {"e4m3": torch.float8_e4m3fn, "int8": torch.int8}


def angles(pos, freq):
    """Angles in radians [tokens, pairs] of integer positions; freq: turns times 2^64
    (Python integers), so that the fraction of a turn is exact."""
    t = [[(int(p) * int(f)) % (1 << 64) for f in freq] for p in pos]
    return torch.tensor([[x / 2.0 ** 64 for x in row] for row in t], dtype=torch.float64).reshape(len(pos), len(freq)) * (2 * np.pi)


def rotate(x, pos, freq, rot, pairs, amp=1.0, back=False):
    """x [tokens, heads, d] -> (rotated, bound).  cos, sin are rounded to fp32, each
    product and the sum once: 3 fp32 roundings of |a cos| + |b sin|; angles in double
    and sines to 2^-45 add less than one more."""
    x = x.double()
    a = angles(pos, freq)
    c, s = amp * torch.cos(a)[:, None], amp * torch.sin(a)[:, None] * (-1 if back else 1)
    i = torch.arange(rot // 2)
    p, q = (2 * i, 2 * i + 1) if pairs else (i, i + rot // 2)
    y, t = x.clone(), torch.zeros_like(x)
    y[..., p], y[..., q] = x[..., p] * c - x[..., q] * s, x[..., p] * s + x[..., q] * c
    t[..., p] = 4 * F32 * ((x[..., p] * c).abs() + (x[..., q] * s).abs())
    t[..., q] = 4 * F32 * ((x[..., p] * s).abs() + (x[..., q] * c).abs())
    return y, t


def scale_of(amax, fmt):
    """The smallest power of two s in 2^-64 .. 2^112 with amax <= top s."""
    e = -64
    while e < 112 and amax > TOP[fmt] * 2.0 ** e:
        e += 1
    return 2.0 ** e


def encode(x, fmt):
    """Values on their scale (fp32) -> codes (uint8 bits)."""
    x = torch.nan_to_num(x, nan=0.0, posinf=3e38, neginf=-3e38)
    if fmt == "int8":
        return torch.round(x.clamp(-127, 127)).to(torch.int8).view(torch.uint8)
    return x.clamp(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8)


def decode(codes, fmt):
    return codes.view(DTYPE[fmt]).to(torch.float32)


class Cache:
    """One layer's cache on the CPU, with the library's layout."""

    def __init__(self, pages, kvh, d, fmt, fill):
        self.K = torch.full((pages, kvh, PAGE, d), fill, dtype=torch.uint8)
        self.V = torch.full((pages, kvh, d, PAGE), fill, dtype=torch.uint8)
        self.scales = torch.full((pages, kvh, 2), 3.0)
        self.fmt = fmt

    def write(self, row, start, K, V):
        """Tokens K, V [n, kvh, d] (fp32 values) at positions start .. of a sequence
        whose pages are `row`; a page at a time, as one call does it."""
        n = K.shape[0]
        for page in range(start // PAGE, -(-(start + n) // PAGE)):
            lo, hi = max(start - page * PAGE, 0), min(start + n - page * PAGE, PAGE)
            r = slice(page * PAGE + lo - start, page * PAGE + hi - start)
            p = int(row[page])
            if not 0 <= p < self.K.shape[0]:
                continue
            for h in range(K.shape[1]):
                for j, (x, buf) in enumerate(((K[r, h], self.K[p, h]), (V[r, h].t(), self.V[p, h]))):
                    ok = x[torch.isfinite(x)]
                    s = scale_of(float(ok.abs().max()) if ok.numel() else 0.0, self.fmt)
                    old, new = (buf[:lo], buf[lo:hi]) if j == 0 else (buf[:, :lo], buf[:, lo:hi])
                    if lo > 0:
                        was = float(self.scales[p, h, j])
                        s = max(s, was)
                        old.copy_(encode(decode(old.contiguous(), self.fmt) * (was / s), self.fmt))
                    new.copy_(encode((x.double() / s).float().contiguous(), self.fmt))
                    self.scales[p, h, j] = s

    def values(self, row, n, pages):
        """float64 K, V [n, kvh, d] of a sequence's first n tokens, and which of them
        lie in a page of the cache."""
        m = -(-n // PAGE)
        p = torch.as_tensor(np.asarray(row[:m], dtype=np.int64))
        there = (p >= 0) & (p < pages)
        p = p.clamp(0, pages - 1)
        k = decode(self.K[p].contiguous(), self.fmt).double() * self.scales[p, :, 0].double()[..., None, None]
        v = decode(self.V[p].contiguous(), self.fmt).double() * self.scales[p, :, 1].double()[..., None, None]
        kvh, d = self.K.shape[1], self.K.shape[3]
        return (k.permute(0, 2, 1, 3).reshape(-1, kvh, d)[:n], v.permute(0, 3, 1, 2).reshape(-1, kvh, d)[:n],
                there.repeat_interleave(PAGE)[:n])


def attention(Q, K, V, there, scale, causal):
    """One sequence: Q [lq, heads, d], K and V [lk, kvh, d] (float64).  Dict of O, lse and
    bounds t_O, t_lse.

    A score is a sum of d exact products in fp32 (d + 16 roundings of sum |q k|), and
    so are the exponents; p is off by their difference and by F16 of itself, or by
    2^-33 of the row's largest; O by BF16 of itself."""
    lq, heads, d = Q.shape
    lk, kvh, _ = K.shape
    G = heads // kvh
    Q = Q.double()
    see = there[None, :].expand(lq, lk).clone()
    if causal:
        see &= torch.arange(lk)[None, :] <= torch.arange(lq)[:, None] + lk - lq
    some = see.any(1)
    z = dict(dtype=torch.float64)
    r = dict(O=torch.zeros((lq, heads, d), **z), lse=torch.full((heads, lq), -np.inf, **z),
             t_O=torch.zeros((lq, heads, d), **z), t_lse=torch.zeros((heads, lq), **z))
    if lk == 0 or lq == 0:
        return r
    for h in range(heads):
        q, k, v = Q[:, h], K[:, h // G], torch.where(there[:, None], V[:, h // G], torch.zeros_like(V[:, 0]))
        k = torch.where(there[:, None], k, torch.zeros_like(k))
        s = (scale * (q @ k.T)).masked_fill(~see, -np.inf)
        m = s.amax(1, keepdim=True)
        m[~some] = 0.0
        w = torch.exp(s - m)
        tot = w.sum(1, keepdim=True)
        p = torch.where(some[:, None], w / tot, torch.zeros_like(w))
        o, pv = p @ v, p @ v.abs()
        zz = (scale * (q.abs() @ k.abs().T)).masked_fill(~see, 0.0).amax(1)
        t_z = (d + 16) * F32 * (zz + 1) + 8 * F32 * (lk + 1) ** 0.5
        r["O"][:, h] = o
        r["t_O"][:, h] = BF16 * o.abs() + (F16 + 3 * t_z[:, None]) * pv + 2.0 ** -33 * v.abs().sum(0)
        r["lse"][h] = torch.where(some, (m + torch.log(tot)).squeeze(1), torch.full((lq,), -np.inf, **z))
        r["t_lse"][h] = t_z
    return r
