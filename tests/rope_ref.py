"""Norms of queries and keys with rotary positions from their definition, in 64 bits on the CPU, with bounds on how far a kernel's
results may be from them.

Outputs are rounded once, by at most eps/2 of their type.  Ahead of that, in fp32 (2^-24 each): the sum of d <= 256 squares (8 in a lane and 5
steps across lanes: 13), their mean and eps (2), half of which reach r, the root (2), the products with r and w (2); cos and sin with
their reduced argument (6), the two products and their sum (2): 20 in all, below 2^-19 of |y1| + |y2|.  The angle in turns is rounded twice to
64 bits: 2^-51 of the angle covers that.  Backward: r to the third power and a second sum of 13 make 60 at most, below 2^-18."""
import math

import torch


def f64(t):
    return t.detach().cpu().double()


def angles(pos, freq, axis):
    """[B, n, 1, rot / 2]"""
    axes = pos.shape[0]
    ax = torch.zeros(freq.shape[0], dtype=torch.long) if axis is None else axis.cpu().long().clamp(0, axes - 1)
    return (f64(pos)[ax].permute(1, 2, 0) * f64(freq)).unsqueeze(2)


def pairs(x, rot, interleaved):
    return (x[..., 0:rot:2], x[..., 1:rot:2]) if interleaved else (x[..., :rot // 2], x[..., rot // 2:rot])


def joined(a, b, rest, interleaved):
    return torch.cat([torch.stack([a, b], -1).flatten(-2) if interleaved else torch.cat([a, b], -1), rest], -1)


def turned(y, ang, interleaved, back=False):
    rot = 2 * ang.shape[-1]
    a, b = pairs(y, rot, interleaved)
    c, s = torch.cos(ang), -torch.sin(ang) if back else torch.sin(ang)
    return joined(a * c - b * s, b * c + a * s, y[..., rot:], interleaved)


def both(y, ang, interleaved):
    """|y1| + |y2| at both places of a pair (1 + what the angle's rounding moves), |y| where nothing turns."""
    rot = 2 * ang.shape[-1]
    a, b = (x.abs() for x in pairs(y, rot, interleaved))
    return joined(a + b, a + b, y[..., rot:].abs(), interleaved), joined((a + b) * ang.abs(), (a + b) * ang.abs(), 0 * y[..., rot:], interleaved)


def normed(x, w, eps):
    r = 1 / torch.sqrt((x * x).mean(-1, keepdim=True) + eps)
    return x * r * (1 if w is None else f64(w)), r


def angles_of(x, pos, freq, axis):
    return angles(pos, freq, axis) if freq is not None else torch.zeros(*x.shape[:2], 1, 0).double()   # (nothing turns)


def fwd(x, pos, freq, axis, interleaved, norm, w, eps):
    """[B, heads, n, d] in 64 bits, and its bound."""
    half = torch.finfo(x.dtype).eps / 2
    ang = angles_of(x, pos, freq, axis)
    y = normed(f64(x), w, eps)[0] if norm else f64(x)
    o = turned(y, ang, interleaved)
    m, far = both(y, ang, interleaved)
    return tuple(z.transpose(1, 2) for z in (o, half * o.abs() + 2 ** -19 * m + 2 ** -51 * far + 1e-37))


def bwd(x, pos, freq, axis, interleaved, norm, w, eps, grad):
    """dx [B, n, heads, d] and dw [d] (None without norm) in 64 bits, and their bounds; grad [B, heads, n, d]."""
    half = torch.finfo(x.dtype).eps / 2
    ang = angles_of(x, pos, freq, axis)
    g = f64(grad).transpose(1, 2)
    m, far = both(g, ang, interleaved)
    g = turned(g, ang, interleaved, back=True)
    lost = 2 ** -18 * m + 2 ** -51 * far
    if not norm:
        return g, None, half * g.abs() + lost + 1e-37, None
    xd = f64(x)
    w = torch.ones(x.shape[-1]).double() if w is None else f64(w)
    r = normed(xd, None, eps)[1]
    dx = r * (w * g) - xd * r ** 3 * (xd * w * g).mean(-1, keepdim=True)
    bound = half * dx.abs() + r * w.abs() * lost + xd.abs() * r ** 3 * (xd.abs() * w.abs() * (lost + 2 ** -18 * m)).mean(-1, keepdim=True) + 1e-37
    dw = (xd * r * g).sum((0, 1, 2))
    # sums of fp32: a lane's rows one after another (every head of its tokens, 2048 groups of tokens at once), then the tokens of a group (256 lanes,
    # of which a row has one for 8 channels, a power of two of them)
    B, n, heads, d = x.shape
    group = 256 // 2 ** math.ceil(math.log2(d / 8))
    steps = heads * -(-(-(-B * n // group)) // 2048) + group + 4
    wb = 2 ** -24 * steps * (xd.abs() * r * m).sum((0, 1, 2)) + (xd.abs() * r * lost).sum((0, 1, 2)) + 2 ** -24 * dw.abs() + 1e-37
    return dx, dw, bound, wb
