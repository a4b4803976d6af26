"""Attention over selected blocks of 64 tokens and the cache in 8 bits from their definitions, in 64 bits on the CPU, with bounds
on how far a kernel's results may be from them.

A value rounded to bf16 is off by at most 2^-8 of itself (half a step), one rounded to fp16 by 2^-11.  The kernels round every
output once to bf16; the weights p to fp16 in the forward and over the cache and to bf16 in the backward; the score gradients ds to
fp16 for dq and to the sum of two bf16 numbers for dk; partial results to fp16 relative to the largest value of their block.  Sums
are fp32 (d products of 2^-24 each; 2^-14 covers them and the exponentials with room, for logits below 2^5)."""
import numpy as np
import torch

T = 64
TINY = 2.0 ** -100


def f64(t):
    return t.detach().to("cpu").double()


def codes_i8(x):
    """[.., d] fp32 -> whole numbers (fp32) and scales, in the operations that the definition names (each rounded to fp32)."""
    x = x.float()
    top = x.abs().amax(-1, keepdim=True)
    some = top >= TINY
    f = torch.where(some, torch.ones(()) / torch.where(some, top, torch.ones(())) * torch.tensor(127.0), torch.zeros(()))
    return torch.round(x * f).clamp(-127, 127), torch.where(some, top * (torch.ones(()) / torch.tensor(127.0)), torch.zeros(()))[..., 0]


def mean_codes(blocks):
    """[.., 64, d] -> codes and scales of the mean key."""
    return codes_i8((f64(blocks).sum(-2) / T).float())


def top_of(score, allowed, top):
    """The places of the `top` largest allowed scores of a row, ascending, padded with -1; of equal ones the first."""
    order = sorted((j for j in range(len(score)) if allowed[j]), key=lambda j: (-float(score[j]), j))[:top]
    return sorted(order) + [-1] * (top - len(order))


def select(q, k, top):
    B, H, n, d = q.shape
    Hkv = k.shape[1]
    p8, _ = codes_i8(f64(q).view(B, Hkv, H // Hkv, n, d).sum(2).float())
    nb = n // T
    m8, ms = mean_codes(k[:, :, :nb * T].reshape(B, Hkv, nb, T, d))
    score = (p8.double() @ m8.double().transpose(-1, -2)).float() * ms.unsqueeze(-2)
    idx = torch.full((B, Hkv, n, top), -1, dtype=torch.int32)
    for b in range(B):
        for g in range(Hkv):
            for i in range(n):
                idx[b, g, i] = torch.tensor(top_of(score[b, g, i], [j < i // T for j in range(nb)], top), dtype=torch.int32)
    return idx


def seen(idx, n):
    """[n, n] which keys every query of one key/value head attends."""
    see = np.zeros((n, -(-n // T) * T), bool)
    for i in range(n):
        for j in set(int(x) for x in idx[i]):
            if 0 <= j < i // T:
                see[i, j * T:(j + 1) * T] = True
        see[i, i // T * T:i + 1] = True
    return torch.from_numpy(see[:, :n])


def attn(q, k, v, idx, scale):
    """o, lse, mass in 64 bits and the bounds of o and lse."""
    B, H, n, d = q.shape
    Hkv, nb = k.shape[1], -(-n // T)
    q, k, v = f64(q), f64(k), f64(v)
    o, lse, mass = torch.zeros(B, H, n, d).double(), torch.zeros(B, H, n).double(), torch.zeros(B, Hkv, nb).double()
    ob, lb = torch.zeros_like(o), torch.zeros_like(lse)
    for b in range(B):
        for g in range(Hkv):
            see = seen(idx[b, g].cpu().numpy(), n)
            for h in range(g * (H // Hkv), (g + 1) * (H // Hkv)):
                s = (q[b, h] @ k[b, g].T * scale).masked_fill(~see, -np.inf)
                lse[b, h] = torch.logsumexp(s, 1)
                p = torch.exp(s - lse[b, h][:, None])
                o[b, h] = p @ v[b, g]
                ob[b, h] = 2 ** -8 * o[b, h].abs() + (2 ** -11 + 2 ** -11 + 2 ** -14) * (p @ v[b, g].abs()) + 2 ** -22 * v[b, g].abs().max()
                lb[b, h] = 2 ** -17 * (q[b, h].abs() @ k[b, g].abs().T * scale).masked_fill(~see, 0).amax(1) + 2 ** -20
                mass[b, g] += torch.nn.functional.pad(p.sum(0), (0, nb * T - n)).view(nb, T).sum(1)
    return o, lse, mass, ob, lb


def attn_bwd(q, k, v, idx, o, lse, dO, scale):
    """(dq, dk, dv) in 64 bits and their bounds, for the o and lse that the backward is given."""
    B, H, n, d = q.shape
    Hkv = k.shape[1]
    q, k, v, o, lse, dO = (f64(x) for x in (q, k, v, o, lse, dO))
    dq, dk, dv = torch.zeros_like(q), torch.zeros_like(k), torch.zeros_like(v)
    aq, ak, av = torch.zeros_like(q), torch.zeros_like(k), torch.zeros_like(v)
    for b in range(B):
        for g in range(Hkv):
            see = seen(idx[b, g].cpu().numpy(), n)
            for h in range(g * (H // Hkv), (g + 1) * (H // Hkv)):
                p = torch.exp((q[b, h] @ k[b, g].T * scale).masked_fill(~see, -np.inf) - lse[b, h][:, None])
                dp, delta = dO[b, h] @ v[b, g].T, (dO[b, h] * o[b, h]).sum(1, keepdim=True)
                ds = p * (dp - delta) * scale
                # what the sums behind ds lose, of dp and delta, and of p; then ds is rounded, to two bf16 numbers for dk and to fp16 for dq
                e = 2 ** -14 * ds.abs() + 2 ** -17 * p * (dO[b, h].abs() @ v[b, g].abs().T + (dO[b, h] * o[b, h]).abs().sum(1, keepdim=True)) * scale
                dv[b, g] += p.T @ dO[b, h]
                dk[b, g] += ds.T @ q[b, h]
                dq[b, h] = ds @ k[b, g]
                av[b, g] += (2 ** -8 + 2 ** -14) * p.T @ dO[b, h].abs()
                ak[b, g] += (e + 2 ** -16 * ds.abs()).T @ q[b, h].abs()
                aq[b, h] = (e + (2 ** -11 + 2 ** -11) * ds.abs()) @ k[b, g].abs() + 2 ** -22 * (ds.abs() @ k[b, g].abs()).amax(1, keepdim=True)
    return (dq, dk, dv), tuple(2 ** -8 * x.abs() + a + 1e-30 for x, a in ((dq, aq), (dk, ak), (dv, av)))


# ---- the cache ----

def block_codes(x, fmt):
    """[.., 64, d] -> codes (as values, fp32) and scales."""
    most = 127.0 if fmt == torch.int8 else 448.0
    x = x.detach().cpu().float()
    top = x.abs().amax((-1, -2), keepdim=True)
    some = top >= TINY
    f = torch.where(some, torch.ones(()) / torch.where(some, top, torch.ones(())) * torch.tensor(most), torch.zeros(()))
    y = (x * f).clamp(-most, most)
    y = torch.round(y) if fmt == torch.int8 else y.to(torch.float8_e4m3fn).float()
    return y, torch.where(some, top * (torch.ones(()) / torch.tensor(most)), torch.zeros(()))[..., 0, 0]


def values(t):
    """Codes of either format as fp32 on the CPU."""
    t = t.cpu()
    return t.float() if t.dtype == torch.int8 else t.view(torch.uint8).view(torch.float8_e4m3fn).float()


def row_tokens(cache, lens, b, g):
    """Keys and values [len, d] that sequence b's head g has, in 64 bits, and the place of each one's block."""
    n = max(0, min(int(lens[b]), cache.cap * T + T - 1))
    whole, rest = divmod(n, T)
    pages = cache.table[b, g, :whole].cpu().long()
    ok = (pages >= 0) & (pages < cache.k8.shape[0])
    pages = pages[ok]
    K = values(cache.k8)[pages].double() * cache.ks.cpu()[pages].double().view(-1, 1, 1)
    V = (values(cache.v8)[pages].double() * cache.vs.cpu()[pages].double().view(-1, 1, 1)).transpose(1, 2)
    at = torch.arange(whole)[ok].repeat_interleave(T)
    return (torch.cat([K.reshape(-1, cache.d), f64(cache.kt[b, g, :rest])]), torch.cat([V.reshape(-1, cache.d), f64(cache.vt[b, g, :, :rest]).T]),
            torch.cat([at, torch.full((rest,), whole)]), whole, rest)


def cache_attn(cache, lens, q, idx=None):
    """o, lse, what joins the masses, and the bounds of o."""
    B, H, d = q.shape
    Hkv, G = cache.Hkv, H // cache.Hkv
    scale = cache.cfg.softmax_scale
    o, ob, lse, mass = torch.zeros(B, H, d).double(), torch.zeros(B, H, d).double(), torch.full((B, H), -np.inf).double(), torch.zeros(B, Hkv, cache.cap + 1).double()
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
                p = torch.exp(s - lse[b, h])
                o[b, h] = p @ V
                ob[b, h] = 2 ** -8 * o[b, h].abs() + (2 ** -11 + 2 ** -14) * (p @ V.abs()) + 1e-30
                mass[b, g].index_add_(0, at, p)
    return o, lse, mass[:, :, :cache.cap], ob


def evict(table, mass, lens, budget, sink, recent):
    table, mass, lens = table.cpu().clone(), mass.cpu().clone(), lens.cpu().clone()
    B, Hkv, cap = table.shape
    for b in range(B):
        nb, rest = divmod(max(0, min(int(lens[b]), cap * T + T - 1)), T)
        lens[b] = min(nb, budget) * T + rest
        if nb <= budget:
            continue
        for g in range(Hkv):
            m = mass[b, g].tolist()
            always = [j < sink or j >= nb - recent for j in range(nb)]
            order = sorted(range(nb), key=lambda j: (not always[j], -m[j] if not always[j] else 0, j))
            kept = sorted(order[:budget])
            gone = sorted(order[budget:])
            table[b, g] = table[b, g][torch.tensor(kept + gone + list(range(nb, cap)), dtype=torch.long)]
            new = [m[j] for j in kept] + [m[nb] if nb < cap else 0.0]
            mass[b, g] = torch.tensor((new + [0.0] * cap)[:cap])
    return table, mass, lens
