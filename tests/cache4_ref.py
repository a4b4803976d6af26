"""The cache in 4 bits from its definition, in 64 bits on the CPU.

Bounds of the attention are those of the cache in 8 bits: outputs are rounded once to bf16 (2^-8), weights to fp16 (2^-11), values are exact in
fp16 relative to their page, sums are fp32 (2^-14 covers them and the exponentials with room, for logits below 2^5)."""
import math

import numpy as np
import torch

from block_ref import T, TINY, f64, mean_codes  # noqa: F401

MAGNITUDES = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def exponent(top):
    """The smallest e with top <= 6 * 2^e, at most 125; None below 2^-100."""
    if top < TINY:
        return None
    e = math.frexp(top / 6.0)[1] - 2
    while top > 6.0 * 2.0 ** e:
        e += 1
    return min(e, 125)


def code(y):
    """The nearest code of y >= 0; of two the even one; 6 at most."""
    y = min(y, 6.0)
    near = sorted(range(8), key=lambda c: (abs(MAGNITUDES[c] - y), c % 2))
    return near[0]


def group(x):
    """32 values: codes, biased exponent, and the values that they stand for."""
    e = exponent(max(abs(float(v)) for v in x))
    if e is None:
        return [0] * 32, 0, [0.0] * 32
    codes = [code(abs(float(v)) / 2.0 ** e) | (8 if math.copysign(1.0, float(v)) < 0 else 0) for v in x]
    return codes, e + 127, [(-1 if c & 8 else 1) * MAGNITUDES[c & 7] * 2.0 ** e for c in codes]


def page_bytes(keys, vals):
    """k4, v4, ke, ve of a block [64, d], from where the header says that they lie."""
    d = keys.shape[1]
    W, two = d // 4, 128 // d
    k4, v4 = np.zeros(32 * d, np.uint8), np.zeros(32 * d, np.uint8)
    ke, ve = np.zeros(2 * d, np.uint8), np.zeros(2 * d, np.uint8)
    for s in range(T):
        a, t, r = s // 16, s // 4 % 4, s % 4
        for j in range(d // 32):
            codes, e, _ = group(keys[s, 32 * j:32 * j + 32].tolist())
            ke[np.ravel_multi_index((j, a, r, t), (d // 32, 4, 4, 4))] = e
            for x, c in enumerate(codes):
                g, i = divmod(32 * j + x, W)
                at = np.ravel_multi_index((t // two, g, a, r, t % two, i), (4 // two, 4, 4, 4, two, W))
                k4[at // 2] |= c << 4 * (at % 2)
    for c in range(d):
        for j in range(2):
            codes, e, _ = group(vals[32 * j:32 * j + 32, c].tolist())
            ve[np.ravel_multi_index((j, c % 16, c // 16), (2, 16, d // 16))] = e
            for x, y in enumerate(codes):
                s = 32 * j + x
                at = np.ravel_multi_index((c // 32, s // 16, c % 16, c // 16 % 2, s % 16), (d // 32, 4, 16, 2, 16))
                v4[at // 2] |= y << 4 * (at % 2)
    return tuple(torch.from_numpy(x) for x in (k4, v4, ke, ve))


def page_scale(e):
    """What ks or vs holds for a page's biased exponents."""
    top = int(e.max())
    low = min((int(x) for x in e.tolist() if x), default=0)
    return 2.0 ** (top - 127) * (1.5 if low < top - 36 else 1.0) if top else 0.0


def rounded(x, dim):
    """[.., 64, d] -> the values that a block stands for, in 64 bits; dim: along which 32 share a scale (-1: keys, -2: values)."""
    y = f64(x).movedim(dim, -1)
    flat = y.reshape(-1, 32)
    top = flat.abs().amax(1, keepdim=True)
    e = torch.tensor([[exponent(float(v))] if v >= TINY else [-1000] for v in top[:, 0]], dtype=torch.float64)
    unit = torch.where(e > -1000, 2.0 ** e.clamp(min=-200), torch.ones(()).double())
    a = (flat.abs() / unit).clamp(max=6)
    step = torch.where(a < 2, 0.5, torch.where(a < 4, 1.0, 2.0)).double()
    z = torch.where(e > -1000, torch.round(a / step) * step * unit * torch.where(flat < 0, -1.0, 1.0), torch.zeros(()).double())
    return z.view(y.shape).movedim(-1, dim)


def dequantised(cache, page):
    """Keys and values [64, d] of a page, from its bytes."""
    d = cache.d
    two, lut = 128 // d, torch.tensor([*MAGNITUDES, *(-x for x in MAGNITUDES)], dtype=torch.float64)
    nib = lambda x: torch.stack([x & 15, x >> 4], -1).flatten()   # noqa: E731
    exp = lambda x: torch.where(x > 0, 2.0 ** (x.double() - 127), torch.zeros(()).double())   # noqa: E731
    k = lut[nib(cache.k4[page].cpu()).long()].view(4 // two, 4, 4, 4, two, d // 4).permute(2, 0, 4, 3, 1, 5).reshape(T, d)
    e = exp(cache.ke[page].cpu()).view(d // 32, 4, 4, 4).permute(1, 3, 2, 0).reshape(T, d // 32)
    v = lut[nib(cache.v4[page].cpu()).long()].view(d // 32, 4, 16, 2, 16).permute(1, 4, 0, 3, 2).reshape(T, d)
    f = exp(cache.ve[page].cpu()).view(2, 16, d // 16).permute(0, 2, 1).reshape(2, d)
    nan = lambda s: float("nan") if math.isnan(float(s)) else 1.0   # noqa: E731
    return k * e.repeat_interleave(32, 1) * nan(cache.ks[page]), v * f.repeat_interleave(32, 0) * nan(cache.vs[page])


def row_tokens(cache, lens, b, g):
    """Keys and values [len, d] that sequence b's head g has, and the place of each one's block."""
    n = max(0, min(int(lens[b]), cache.cap * T + T - 1))
    whole, rest = divmod(n, T)
    K, V, at = [], [], []
    for j in range(whole):
        page = int(cache.table[b, g, j])
        if 0 <= page < cache.k4.shape[0]:
            k, v = dequantised(cache, page)
            K.append(k)
            V.append(v)
            at += [j] * T
    K.append(f64(cache.kt[b, g, :rest]))
    V.append(f64(cache.vt[b, g, :, :rest]).T)
    return torch.cat(K), torch.cat(V), torch.tensor(at + [whole] * rest, dtype=torch.long), whole, rest


def cache_attn(cache, lens, q, idx=None):
    """o, lse, what joins the masses, and the bounds of o."""
    B, H, d = q.shape
    Hkv, G, scale = cache.Hkv, H // cache.Hkv, cache.cfg.softmax_scale
    o, ob, lse = torch.zeros(B, H, d).double(), torch.zeros(B, H, d).double(), torch.full((B, H), -np.inf).double()
    mass = torch.zeros(B, Hkv, cache.cap + 1).double()
    q = f64(q)
    for b in range(B):
        for g in range(Hkv):
            K, V, at, whole, rest = row_tokens(cache, lens, b, g)
            if idx is not None:
                own = whole if rest else whole - 1
                keep = torch.zeros(cache.cap + 2, dtype=torch.bool)
                for j in idx[b, g].tolist():
                    if 0 <= j < own:
                        keep[j] = True
                keep[own] = True
                K, V, at = K[keep[at]], V[keep[at]], at[keep[at]]
            if len(at) == 0:
                continue
            for h in range(g * G, (g + 1) * G):
                s = K @ q[b, h] * scale
                lse[b, h] = torch.logsumexp(s, 0)
                p = torch.softmax(s, 0)   # (not exp(s - lse): of logits beyond 2^52 the logarithm of a count is lost in 64 bits)
                o[b, h] = p @ V
                ob[b, h] = 2 ** -8 * o[b, h].abs() + (2 ** -11 + 2 ** -14) * (p @ V.abs()) + 1e-30
                mass[b, g].index_add_(0, at, p)
    return o, lse, mass[:, :, :cache.cap], ob
